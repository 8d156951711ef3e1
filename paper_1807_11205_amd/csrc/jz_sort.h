// Positions sorted by token, stably: least significant digits first, up to nine bits a pass.  Included inside a kernel file's anonymous namespace.
//
// A token outside [0, vocab) gets the key `vocab` and so comes last.  Within a wavefront equal digits find each other by ballots, a lane's rank among them is the
// number of lower lanes with its digit, and a counter for each wavefront and digit carries the count from one 64 to the next: no order depends on who comes first.
// Up to 16384 tokens are sorted as runs of 1024 in LDS, and the runs joined: two launches.  (One workgroup for all of them was bound by what one compute unit can do: 16384 tokens of 50000, 35 us by
// ballots, 46 with counters for each thread and digit.)  Beyond, each pass is three launches: counts of the digits in tiles of 4096, their running sums over the tiles, and the
// move; counts and moves are n / 4096 workgroups, so that short ones leave most of the chip idle (20000 tokens of 100000 x 64, two passes: 83 us for gradient and lookup, of 500 x 64, one pass: 57).
// On the way `used` (one byte for each token of the vocabulary, or NULL) is cleared and then set where a token occurs, and *counter is cleared.
#pragma once

constexpr int SORT_BITS = 9, SORT_RADIX = 1 << SORT_BITS, SORT_TILE = 4096;
constexpr int64_t SORT_SMALL = 16384;

struct SortLayout {
  int all_bits, passes, bits;  // of a key; passes of the large form and bits of their digits
  int64_t tiles;
  size_t keys[2], pos[2], counts, totals, total;
};
inline SortLayout sort_layout(int64_t n, int vocab) {
  SortLayout L;
  int bits = 1;
  while (bits < 32 && (int64_t(1) << bits) <= vocab) ++bits;  // the largest key is `vocab`
  L.all_bits = bits;
  L.passes = (bits + SORT_BITS - 1) / SORT_BITS;
  L.bits = (bits + L.passes - 1) / L.passes;
  L.tiles = n > SORT_SMALL ? (n + SORT_TILE - 1) / SORT_TILE : 0;
  size_t o = 0;
  auto room = [&](size_t bytes) {
    const size_t at = o;
    o = (o + bytes + 255) & ~size_t(255);
    return at;
  };
  const size_t list = (size_t)n * 4;
  L.keys[0] = room(list);
  L.pos[0] = room(list);
  L.keys[1] = n > 1024 ? room(list) : 0;
  L.pos[1] = n > 1024 ? room(list) : 0;
  L.counts = room((size_t)L.tiles * SORT_RADIX * 4);
  L.totals = room(L.tiles ? SORT_RADIX * 4 : 0);
  L.total = o;
  return L;
}

struct SortArgs {
  const int* ids;
  const unsigned *keys_in, *pos_in;  // or the ids themselves, in the first pass
  unsigned *keys, *pos, *counts, *totals, *counter;
  unsigned char* used;               // cleared in the first pass, set in the last
  int64_t n, tiles;
  int vocab, shift, bits, all_bits;
  bool first, last;
};

__device__ __forceinline__ unsigned sort_key(int id, int vocab) { return (unsigned)id < (unsigned)vocab ? (unsigned)id : (unsigned)vocab; }

// A lane's rank among the keys with its digit that its wavefront has had, this 64 included.
__device__ __forceinline__ unsigned rank_in_wave(unsigned digit, int bits, unsigned* count) {
  unsigned long long same = ~0ull;
  for (int b = 0; b < bits; ++b) {
    const bool on = digit >> b & 1;
    const unsigned long long with = __ballot(on);
    same &= on ? with : ~with;
  }
  const int lane = threadIdx.x & 63, leader = __ffsll((long long)same) - 1;
  const unsigned before = __popcll(same & ((1ull << lane) - 1));
  unsigned old = 0;
  if (lane == leader) old = atomicAdd(count + digit, (unsigned)__popcll(same));
  return __shfl(old, leader) + before;
}

// Running sum over the workgroup's threads of one value each; lds: one word a wavefront.
template <int WAVES>
__device__ __forceinline__ unsigned exclusive_sum(unsigned v, unsigned* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  unsigned s = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const unsigned up = __shfl_up(s, d);
    if (lane >= d) s += up;
  }
  if (lane == 63) lds[wave] = s;
  __syncthreads();
  unsigned base = 0;
  for (int w = 0; w < wave && w < WAVES; ++w) base += lds[w];
  __syncthreads();
  return base + s - v;
}

// Runs of 1024 positions, a workgroup each, one key a thread: sorted by itself in LDS.  Keys behind the last are the largest there are and stay behind it.
__global__ __launch_bounds__(1024) void sort_runs(SortArgs a) {
  __shared__ unsigned keys[1024], pos[1024];
  __shared__ unsigned count[16][SORT_RADIX], start[SORT_RADIX], scan[16];
  const int t = threadIdx.x, wave = t >> 6, radix = 1 << a.bits;
  const int64_t i = (int64_t)blockIdx.x * 1024 + t;
  unsigned k = i < a.n ? sort_key(a.ids[i], a.vocab) : ~0u, p = (unsigned)i;
  if (a.used)
    for (int64_t u = i * 16; u < a.vocab; u += (int64_t)gridDim.x * 1024 * 16) *reinterpret_cast<uint4*>(a.used + u) = uint4{0, 0, 0, 0};  // whole: its room ends on 256 bytes
  if (i == 0) *a.counter = 0;
  for (int shift = 0; shift < a.all_bits; shift += a.bits) {
    for (int c = t; c < 16 * radix; c += 1024) count[c >> a.bits][c & (radix - 1)] = 0;
    __syncthreads();
    const unsigned d = k >> shift & (radix - 1), r = rank_in_wave(d, a.bits, count[wave]);
    __syncthreads();
    unsigned all = 0;
    if (t < radix) {
      unsigned c[16];
#pragma unroll
      for (int w = 0; w < 16; ++w) c[w] = count[w][t];
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        count[w][t] = all;
        all += c[w];
      }
    }
    const unsigned before = exclusive_sum<16>(all, scan);
    if (t < radix) start[t] = before;
    __syncthreads();
    const unsigned to = start[d] + count[wave][d] + r;
    keys[to] = k;
    pos[to] = p;
    __syncthreads();
    k = keys[t];
    p = pos[t];
  }
  if (i < a.n) {
    a.keys[i] = k;
    a.pos[i] = p;
    if (a.tiles == 1 && a.used && k < (unsigned)a.vocab) a.used[k] = 1;  // one run: this workgroup alone has cleared it, before the barriers above
  }
}

// Up to RUNS runs into one list: a key's place is its place in its run and the number of keys before it in each other run, by bisection; equal keys of earlier runs come first.
template <int RUNS>
__global__ __launch_bounds__(256) void sort_merge(SortArgs a) {
  __shared__ __attribute__((aligned(16))) unsigned keys[RUNS * 1024];
  const int runs = (int)a.tiles, t = threadIdx.x;
  const int64_t i = (int64_t)blockIdx.x * 256 + t;
  const unsigned mine = i < a.n ? a.keys_in[i] : ~0u, p = i < a.n ? a.pos_in[i] : 0;
  const int n = (int)a.n, end = (n - 1) & ~3;  // the last four there are: a list's room ends on 256 bytes
  uint4 v[RUNS];
#pragma unroll
  for (int j = 0; j < RUNS; ++j) {  // asked for together
    const int at = j * 1024 + t * 4;
    v[j] = *reinterpret_cast<const uint4*>(a.keys_in + (at < end ? at : end));
  }
#pragma unroll
  for (int j = 0; j < RUNS; ++j) {
    const int at = j * 1024 + t * 4;
    if (at >= n) v[j].x = ~0u;
    if (at + 1 >= n) v[j].y = ~0u;
    if (at + 2 >= n) v[j].z = ~0u;
    if (at + 3 >= n) v[j].w = ~0u;
    *reinterpret_cast<uint4*>(keys + at) = v[j];
  }
  __syncthreads();
  if (i >= a.n) return;
  const int run = (int)(i >> 10);
  unsigned to = (unsigned)(i & 1023);
  constexpr int Q = RUNS < 8 ? RUNS : 8;  // bisections at a time
  for (int q0 = 0; q0 < runs; q0 += Q) {
    unsigned at[Q] = {};
#pragma unroll
    for (int s = 512; s > 0; s >>= 1)
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const int of = q0 + q < runs ? q0 + q : 0;
        if (keys[of * 1024 + at[q] + s - 1] < mine + (of < run ? 1u : 0u)) at[q] += s;
      }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int of = q0 + q;
      if (of >= runs || of == run) continue;
      if (keys[of * 1024 + at[q]] < mine + (of < run ? 1u : 0u)) ++at[q];
      to += at[q];
    }
  }
  a.keys[to] = mine;
  a.pos[to] = p;
  if (a.used && mine < (unsigned)a.vocab) a.used[mine] = 1;
}

__global__ __launch_bounds__(256) void sort_count(SortArgs a) {
  __shared__ unsigned count[SORT_RADIX];
  const int radix = 1 << a.bits;
  for (int i = threadIdx.x; i < radix; i += 256) count[i] = 0;
  if (a.first) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.counter = 0;
    if (a.used)
      for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 16; i < a.vocab; i += (int64_t)gridDim.x * 256 * 16)
        *reinterpret_cast<uint4*>(a.used + i) = uint4{0, 0, 0, 0};
  }
  __syncthreads();
  const int64_t at = (int64_t)blockIdx.x * SORT_TILE;
#pragma unroll 4
  for (int j = 0; j < SORT_TILE / 256; ++j) {
    const int64_t i = at + j * 256 + threadIdx.x;
    if (i < a.n) atomicAdd(&count[(a.first ? sort_key(a.ids[i], a.vocab) : a.keys_in[i]) >> a.shift & (radix - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < radix; i += 256) a.counts[(int64_t)i * a.tiles + blockIdx.x] = count[i];
}

// one workgroup a digit: what its tiles before have of it, and all of them
__global__ __launch_bounds__(256) void sort_scan(SortArgs a) {
  __shared__ unsigned scan[4];
  __shared__ unsigned last;
  unsigned* const c = a.counts + (int64_t)blockIdx.x * a.tiles;
  unsigned carry = 0;
  for (int64_t at = 0; at < a.tiles; at += 256) {
    const int64_t i = at + threadIdx.x;
    const unsigned v = i < a.tiles ? c[i] : 0, before = exclusive_sum<4>(v, scan);
    if (i < a.tiles) c[i] = carry + before;
    if (threadIdx.x == 255) last = before + v;
    __syncthreads();
    carry += last;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.totals[blockIdx.x] = carry;
}

__global__ __launch_bounds__(256) void sort_move(SortArgs a) {
  constexpr int EACH = SORT_TILE / 256;
  __shared__ unsigned count[4][SORT_RADIX], scan[4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, radix = 1 << a.bits;
  const int64_t at = (int64_t)blockIdx.x * SORT_TILE + wave * (64 * EACH) + lane;
  unsigned k[EACH], p[EACH], r[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int64_t i = at + j * 64;
    k[j] = ~0u;
    p[j] = (unsigned)i;
    if (i < a.n) {
      k[j] = a.first ? sort_key(a.ids[i], a.vocab) : a.keys_in[i];
      if (!a.first) p[j] = a.pos_in[i];
    }
  }
  for (int i = t; i < 4 * SORT_RADIX; i += 256) count[i / SORT_RADIX][i % SORT_RADIX] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) r[j] = rank_in_wave(k[j] >> a.shift & (radix - 1), a.bits, count[wave]);  // keys behind the last come last of all
  // where each digit's keys begin: two digits a thread, in order
  const unsigned d0 = 2 * t, d1 = 2 * t + 1;
  const unsigned c0 = d0 < (unsigned)radix ? a.totals[d0] : 0, c1 = d1 < (unsigned)radix ? a.totals[d1] : 0;
  __syncthreads();
  const unsigned before = exclusive_sum<4>(c0 + c1, scan);
  auto place = [&](unsigned d, unsigned from) {
    if (d >= (unsigned)radix) return;
    unsigned b = from + a.counts[(int64_t)d * a.tiles + blockIdx.x];
    for (int w = 0; w < 4; ++w) {
      const unsigned c = count[w][d];
      count[w][d] = b;
      b += c;
    }
  };
  place(d0, before);
  place(d1, before + c0);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    if (at + j * 64 >= a.n) continue;
    const unsigned to = count[wave][k[j] >> a.shift & (radix - 1)] + r[j];
    a.keys[to] = k[j];
    a.pos[to] = p[j];
    if (a.last && a.used && k[j] < (unsigned)a.vocab) a.used[k[j]] = 1;
  }
}

// n > 0 ids (or none: `used` and the counter alone) -> sorted keys and positions inside the workspace `b`
inline int sort_tokens(const SortLayout& L, const int* ids, int64_t n, int vocab, unsigned char* used, unsigned* counter, char* b, const unsigned** keys, const unsigned** pos,
                       hipStream_t st) {
  auto list = [&](size_t at) { return reinterpret_cast<unsigned*>(b + at); };
  SortArgs a = {};
  a.ids = ids;
  a.n = n;
  a.tiles = L.tiles;
  a.vocab = vocab;
  a.bits = L.bits;
  a.all_bits = L.all_bits;
  a.used = used;
  a.counter = counter;
  a.counts = list(L.counts);
  a.totals = list(L.totals);
  if (n <= SORT_SMALL) {
    const unsigned runs = (unsigned)std::max<int64_t>(1, (n + 1023) / 1024);
    a.tiles = runs;
    a.keys = list(L.keys[0]);
    a.pos = list(L.pos[0]);
    sort_runs<<<runs, 1024, 0, st>>>(a);
    if (runs > 1) {
      if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
      a.keys_in = a.keys;
      a.pos_in = a.pos;
      a.keys = list(L.keys[1]);
      a.pos = list(L.pos[1]);
      const unsigned grid = (unsigned)((n + 255) / 256);
      if (runs <= 4) sort_merge<4><<<grid, 256, 0, st>>>(a);
      else sort_merge<16><<<grid, 256, 0, st>>>(a);
    }
    *keys = a.keys;
    *pos = a.pos;
    return jz::launch_status();
  }
  for (int pass = 0; pass < L.passes; ++pass) {
    const int to = pass & 1;
    a.first = pass == 0;
    a.last = pass == L.passes - 1;
    a.shift = pass * L.bits;
    a.keys_in = list(L.keys[!to]);
    a.pos_in = list(L.pos[!to]);
    a.keys = list(L.keys[to]);
    a.pos = list(L.pos[to]);
    sort_count<<<(unsigned)L.tiles, 256, 0, st>>>(a);
    sort_scan<<<1u << L.bits, 256, 0, st>>>(a);
    sort_move<<<(unsigned)L.tiles, 256, 0, st>>>(a);
    if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  }
  *keys = a.keys;
  *pos = a.pos;
  return JZ_OK;
}
