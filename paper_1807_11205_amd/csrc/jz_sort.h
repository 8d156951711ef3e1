// Positions sorted by token, stably: least significant digits first, up to nine bits a pass.  Included inside a kernel file's anonymous namespace.
//
// A token outside [0, vocab) gets the key `vocab` and so comes last.  Within a wavefront equal digits find each other by ballots, a lane's rank among them is the
// number of lower lanes with its digit, and a counter for each wavefront and digit carries the count from one 64 to the next: no order depends on who comes first.
// Up to 16384 tokens one workgroup does it all in LDS (one launch; 50000 different tokens are 16 bits, two passes).  Beyond, each pass is three launches: counts of the
// digits in tiles of 4096, their running sums over the tiles, and the move.
// On the way `used` (one byte for each token of the vocabulary, or NULL) is cleared and then set where a token occurs, and *counter is cleared.
#pragma once

constexpr int SORT_BITS = 9, SORT_RADIX = 1 << SORT_BITS, SORT_TILE = 4096;
constexpr int64_t SORT_SMALL = 16384;

struct SortLayout {
  int passes, bits;  // of a digit
  int64_t tiles;
  size_t keys[2], pos[2], counts, totals, total;
};
inline SortLayout sort_layout(int64_t n, int vocab) {
  SortLayout L;
  int bits = 1;
  while (bits < 32 && (int64_t(1) << bits) <= vocab) ++bits;  // the largest key is `vocab`
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
  L.keys[1] = L.tiles ? room(list) : 0;
  L.pos[1] = L.tiles ? room(list) : 0;
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
  int vocab, shift, bits, passes;
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

// Everything in one workgroup: EACH keys a thread, in order: wavefront, turn, lane.  Keys behind the last are the largest there are and stay behind it.
template <int EACH>
__global__ __launch_bounds__(1024) void sort_small(SortArgs a) {
  constexpr int N = 1024 * EACH;
  __shared__ unsigned keys[N];
  __shared__ unsigned short pos[N];
  __shared__ unsigned count[16][SORT_RADIX], start[SORT_RADIX], scan[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, radix = 1 << a.bits;
  unsigned k[EACH], p[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    p[j] = wave * (64 * EACH) + j * 64 + lane;
    k[j] = p[j] < a.n ? sort_key(a.ids[p[j]], a.vocab) : ~0u;
  }
  if (t == 0) *a.counter = 0;
  if (a.used)
    for (int64_t i = (int64_t)t * 16; i < a.vocab; i += 1024 * 16) *reinterpret_cast<uint4*>(a.used + i) = uint4{0, 0, 0, 0};  // whole: its room ends on 256 bytes
  for (int pass = 0; pass < a.passes; ++pass) {
    const int shift = pass * a.bits;
    for (int i = t; i < 16 * SORT_RADIX; i += 1024) count[i / SORT_RADIX][i % SORT_RADIX] = 0;
    __syncthreads();
    unsigned r[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) r[j] = rank_in_wave(k[j] >> shift & (radix - 1), a.bits, count[wave]);
    __syncthreads();
    unsigned all = 0;
    if (t < radix)
      for (int w = 0; w < 16; ++w) {
        const unsigned c = count[w][t];
        count[w][t] = all;
        all += c;
      }
    const unsigned before = exclusive_sum<16>(all, scan);
    if (t < radix) start[t] = before;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const unsigned d = k[j] >> shift & (radix - 1), to = start[d] + count[wave][d] + r[j];
      keys[to] = k[j];
      pos[to] = (unsigned short)p[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int i = wave * (64 * EACH) + j * 64 + lane;
      k[j] = keys[i];
      p[j] = pos[i];
    }
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int i = wave * (64 * EACH) + j * 64 + lane;
    if (i < a.n) {
      a.keys[i] = k[j];
      a.pos[i] = p[j];
      if (a.used && k[j] < (unsigned)a.vocab) a.used[k[j]] = 1;  // cleared before the barriers above
    }
  }
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
  a.passes = L.passes;
  a.used = used;
  a.counter = counter;
  a.counts = list(L.counts);
  a.totals = list(L.totals);
  if (n <= SORT_SMALL) {
    a.keys = list(L.keys[0]);
    a.pos = list(L.pos[0]);
    if (n <= 1024) sort_small<1><<<1, 1024, 0, st>>>(a);
    else if (n <= 4096) sort_small<4><<<1, 1024, 0, st>>>(a);
    else sort_small<16><<<1, 1024, 0, st>>>(a);
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
