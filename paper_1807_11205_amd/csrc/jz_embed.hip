// Embedding lookup and the gradient of its table (include/jz.h: jz_embed_fwd, jz_embed_bwd).
//
//   out[t] = RNE(scale * table[id_t]),      dtable[v] = RNE(scale * sum over t with id_t = v of dout[t]  [+ dtable[v]])
//
// What bounds both: memory.  Forward a table row is read where its token stands and a row is written; backward every row of dout is read once
// and every row of dtable written once.  For that the positions are first sorted by token, stably, so that every sum has one order: first by position.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "jz_internal.h"

namespace {

#include "jz_vec.h"
#include "jz_sort.h"

constexpr int ZERO_EACH = 16384;    // elements of the table that a workgroup looks at
constexpr int EMBED_GRID = 1 << 16;  // workgroups at most: each takes further turns

// Results of STREAM_BYTES and more are written past the caches: the next launch would find little of them there, and the table's rows stay.  Lookup of
// 268 MB in BF16 85.4 us with ordinary stores, 81.0 so, of 262 MB out of 3000 rows 82 and 58, of 134 MB in FP32 43 and 30; the zeros of a table of 205 MB 144.7 and 137.9 with the lookup and all
// (in FP32, two halves of every 32 bytes that go by themselves, 548 and 740: not those).

// ---- lookup -----------------------------------------------------------------------------------------------------------------
struct LookupArgs {
  const int* ids;
  const void* table;
  void* out;
  int64_t tokens, ld;
  int vocab, channels;
  float scale;
};

// Channels that a lane stores at a time: FP32 rows past the caches 16 bytes, since the two halves of 32 would go their ways by themselves.
template <class T, class O>
constexpr int lookup_each(bool stream) {
  return sizeof(O) == 4 && (stream || sizeof(T) == 4) ? 4 : 8;
}
// Groups of EACH channels; a row's last group ends with the row, so that it overlaps its neighbour where channels are no multiple of it (both store the same
// values).  FEW: less than eight channels.  STREAM: past the caches.
template <class T, class O, bool FEW, bool STREAM>
__global__ __launch_bounds__(256) void embed_lookup(LookupArgs a) {
  constexpr int EACH = FEW ? 8 : lookup_each<T, O>(STREAM), U = 32 / EACH;  // U: loads in flight
  typedef T In __attribute__((ext_vector_type(EACH)));
  typedef O Out __attribute__((ext_vector_type(EACH)));
  typedef float F32 __attribute__((ext_vector_type(EACH)));
  typedef In InAny __attribute__((aligned(sizeof(T))));
  typedef Out OutAny __attribute__((aligned(sizeof(O))));
  const int64_t per = (a.channels + EACH - 1) / EACH, all = a.tokens * per;
  const bool small = EACH == 4 && all < int64_t(1) << 32;  // indexes of 32 bits divide faster, which those of 8 hide (84 us for 81 with it)
  for (int64_t base = (int64_t)blockIdx.x * (256 * U); base < all; base += (int64_t)gridDim.x * (256 * U)) {
    In v[U];
    int64_t to[U];
    bool there[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = base + u * 256 + threadIdx.x;
      to[u] = -1;
      there[u] = false;
      v[u] = In{};
      if (i < all) {
        const int64_t t = small ? (unsigned)i / (unsigned)per : i / per;
        int64_t c = (i - t * per) * EACH;
        if (!FEW && c + EACH > a.channels) c = a.channels - EACH;
        const int id = a.ids[t];
        there[u] = (unsigned)id < (unsigned)a.vocab;
        to[u] = t * a.ld + c;
        if (there[u]) {
          const T* p = static_cast<const T*>(a.table) + (int64_t)id * a.channels + c;
          if constexpr (FEW) v[u] = load8(p, a.channels);
          else v[u] = *reinterpret_cast<const InAny*>(p);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (to[u] < 0) continue;
      // a token outside the table: zeros, also with a scale that is not finite
      const Out r = there[u] ? __builtin_convertvector(__builtin_convertvector(v[u], F32) * a.scale, Out) : Out{};
      O* p = static_cast<O*>(a.out) + to[u];
      if constexpr (FEW) store8(p, r, a.channels);
      else if constexpr (STREAM) __builtin_nontemporal_store(r, reinterpret_cast<OutAny*>(p));
      else *reinterpret_cast<OutAny*>(p) = r;
    }
  }
}

typedef f32x4 f32x4_any __attribute__((aligned(4)));

// ---- gradient ---------------------------------------------------------------------------------------------------------------
// The sorted positions are cut into pieces of `piece`.  Where a token's places begin, its piece adds them up, to the end of the next piece at most; if there are more
// of them (a frequent token), every further piece leaves a partial sum of its own, and embed_join adds those up in order.  A thread has eight channels; `lanes`
// threads (a power of two) have a row or, of a wide one, a slice.
//
// Bound: memory.  16384 tokens, 50001 x 2048, FP32 -> FP16: 73 us for 340 MB (4.7 TB/s), 13 us of sorting before and 7 of joining behind; 1777 tokens, 32003 x 1001, BF16: 17 us for 68 MB.
// Blocks that add up come first, those that clear behind them (taking turns: 114 us); 128 registers a lane, so that four workgroups are on a compute unit (without the bound 202: 80 and 24 us).
// Pieces are longer where there are more of them: 8 places, 16 from 4096 tokens and 32 from 32768, that is 256 workers or more from 4096 tokens on and a partial sum for 16 rows or more.  A worker is
// `lanes` threads, a workgroup only where rows are wide: with 64 channels it is 8 of them, 60000 tokens are 59 workgroups, and what bounds such gradients are launches and idle compute units:
// 60000 tokens of 100000 x 64 with the lookup 102 us, 7 of them memory's.
struct SumArgs {
  const unsigned *keys, *pos;   // sorted
  const void* dout;
  void* dtable;
  const unsigned char* used;    // rows of the table that have a token
  float* partial;               // [piece][2][channels]: of a token that began two pieces ago or earlier; of one that goes on behind the next piece
  unsigned *n_long, *long_list; // pieces where such a token begins
  int64_t tokens, ld, pieces;
  int vocab, channels, piece, lanes, slices, accumulate;
  int64_t sum_blocks, zero_blocks;
  float scale;
};

// eight channels from c on of a row, or what there is of them
template <class T>
__device__ __forceinline__ f32x8 row8(const T* p, int left) {
  return widen8<T>(left >= 8 ? load8(p) : load8(p, left));
}

template <class G>
__device__ __forceinline__ void finish_row(const SumArgs& a, unsigned key, int c, int left, f32x8 sum) {
  G* p = static_cast<G*>(a.dtable) + (int64_t)key * a.channels + c;
  f32x8 v = sum * a.scale;
  if (a.accumulate) v += row8(p, left);
  store8(p, narrow8<G>(v), left);
}

// The sorted places of a piece and of the next one, and the tokens before: [0] one place, [1] a piece and one place before.
struct Window {
  unsigned *key, *pos;
  unsigned before[2];
};
template <class O, class G, bool ONCE>
__device__ __forceinline__ void sum_piece(const SumArgs& a, int64_t piece, int c, const Window& w) {
  constexpr int U = sizeof(O) == 4 ? 4 : 8;  // rows on their way at a time
  const int64_t rest = a.tokens - piece * a.piece;
  const int own_end = rest < a.piece ? (int)rest : a.piece, far_end = rest < 2 * a.piece ? (int)rest : 2 * a.piece;
  const int left = a.channels - c < 8 ? a.channels - c : 8;
  int i = 0;
  const unsigned first = w.key[0], last = w.key[own_end - 1];
  if (first >= (unsigned)a.vocab) return;  // tokens outside the table come last
  bool head = false;                       // a token's further part
  if (w.before[0] == first) {
    head = w.before[1] == first;
    if (!head)  // it began in the piece before, which adds this piece's places too
      while (i < own_end && w.key[i] == first) ++i;
  }
  if (i >= own_end) return;
  const bool all_head = head && last == first;  // nothing of the piece is its own: the next piece's places are another's
  const int end = all_head ? own_end : far_end;
  const O* const dout = static_cast<const O*>(a.dout) + c;
  unsigned key = w.key[i];
  f32x8 sum = {};
  auto flush = [&](bool goes_on) {
    if (head || goes_on) {
      store8(a.partial + (piece * 2 + !head) * a.channels + c, sum, left);
      if (!head && c == 0) a.long_list[atomicAdd(a.n_long, 1u)] = (unsigned)piece;  // their order is of no consequence: each has a row of its own
    } else {
      finish_row<G>(a, key, c, left, sum);
    }
    head = false;
  };
  // does the token at the end of what is looked at go on behind it?  (behind two pieces: the place after the window is a third's first)
  auto goes_on = [&](int at) { return at == end && !all_head && rest > end && a.keys[piece * a.piece + end] == key; };
  for (;;) {
    unsigned k[U];
    typename Vec8<O>::V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int at = i + u < end ? i + u : end - 1;
      k[u] = w.key[at];
      const bool mine = i + u < end && k[u] < (unsigned)a.vocab && (i + u < own_end || k[u] == last);
      if (!mine) k[u] = ~0u;
      // in the place of one that is not its own a row that it reads anyway, and does not add
      const O* const p = dout + (int64_t)w.pos[mine ? at : i] * a.ld;
      if constexpr (ONCE) v[u] = left >= 8 ? (typename Vec8<O>::V)__builtin_nontemporal_load(reinterpret_cast<const typename Vec8<O>::U*>(p)) : load8(p, left);
      else v[u] = left >= 8 ? load8(p) : load8(p, left);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k[u] != key) {
        flush(goes_on(i + u));  // what stopped it: another token, the end of the next piece, or of all
        if (k[u] == ~0u) return;
        key = k[u];
        sum = f32x8{};
      }
      sum += widen8<O>(v[u]);
    }
    i += U;
    if (i >= end) {
      flush(goes_on(end));
      return;
    }
  }
}

// STREAM: rows without a token are written past the caches.  ONCE: rows of dout do not stay in them either, where they are half of the last-level cache together, whole lines, and FP32 only in one
// slice, whose halves of lines come at once: 16384 tokens, 50001 x 2048, FP32 134 us without it, 126 so, 60000 of 20000 x 1024 203 and 180, 32000 of 50000 x 4096 in BF16 278 and 272; but 30000 of
// 60000 x 4096 in FP32 425 and 430, of 60000 x 3000 338 and 362, 1777 of 32003 x 1001 in BF16 38.5 and 48.
template <class O, class G, bool STREAM, bool ONCE>
__global__ __launch_bounds__(256, 4) void embed_sum(SumArgs a) {
  __shared__ unsigned keys[32 * 64], pos[32 * 64];  // of each worker: two pieces
  const int per = 256 / a.lanes, mine = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes;
  const int64_t blocks = a.sum_blocks + a.zero_blocks;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    if (b < a.sum_blocks) {
      const int64_t w = b * per + mine, piece = w / a.slices;
      const int c = ((int)(w - piece * a.slices) * a.lanes + lane) * 8;
      const int64_t at = piece * a.piece;
      Window win = {keys + mine * 2 * a.piece, pos + mine * 2 * a.piece, {~0u, ~0u}};
      __syncthreads();  // the previous turn's reads
      if (piece < a.pieces) {
        for (int j = lane; j < 2 * a.piece && at + j < a.tokens; j += a.lanes) {
          win.key[j] = a.keys[at + j];
          win.pos[j] = a.pos[at + j];
        }
        if (piece > 0) win.before[0] = a.keys[at - 1];
        if (piece > 1) win.before[1] = a.keys[at - a.piece - 1];
      }
      __syncthreads();
      if (piece < a.pieces && c < a.channels) sum_piece<O, G, ONCE>(a, piece, c, win);
    } else {  // what lies in rows of the table without a token, in vectors on 16 bytes whatever the channels are
      const int64_t all = (int64_t)a.vocab * a.channels, e0 = (b - a.sum_blocks) * ZERO_EACH, row0 = e0 / a.channels;
      const int n = (int)(all - e0 < ZERO_EACH ? all - e0 : ZERO_EACH);
      const unsigned off = (unsigned)(e0 - row0 * a.channels), D = (unsigned)a.channels;
      G* const to = static_cast<G*>(a.dtable) + e0;
      const unsigned char* const used = a.used + row0;
      constexpr int EACH = ZERO_EACH / (256 * 8);
      unsigned char busy[EACH], next[EACH];  // of the row that a vector begins in, and where one ends inside the vector of the next: does it have a token?  All asked for together
      unsigned ends[EACH];
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const unsigned i = (j * 256 + threadIdx.x) * 8, row = (off + i) / D;
        ends[j] = (row + 1) * D - (off + i);
        busy[j] = (int)i < n ? used[row] : 1;
        next[j] = ends[j] < 8 && (int)(i + ends[j]) < n ? used[row + 1] : 1;
      }
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const int i = (j * 256 + threadIdx.x) * 8;
        if (ends[j] >= 8) {
          if (busy[j]) continue;
          if constexpr (STREAM) stream8(to + i, typename Vec8<G>::V{});
          else store8(to + i, typename Vec8<G>::V{});
        } else if (D >= 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (i + e < n && !(e < (int)ends[j] ? busy[j] : next[j])) to[i + e] = (G)0.f;
        } else {
          for (int e = 0; e < 8 && i + e < n; ++e)
            if (!used[(off + i + e) / D]) to[i + e] = (G)0.f;
        }
      }
    }
  }
}

// The partial sums of a frequent token, added in order: eight wavefronts take an eighth of them each, four channels a lane.
template <class G>
__global__ __launch_bounds__(512) void embed_join(SumArgs a) {
  __shared__ f32x4 sums[8][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned n = *a.n_long;
  for (int64_t c0 = (int64_t)blockIdx.y * 256; c0 < a.channels; c0 += (int64_t)gridDim.y * 256) {
    const int64_t c = c0 + lane * 4;
    const int left = (int)(a.channels - c < 4 ? a.channels - c : 4);
    for (unsigned i = blockIdx.x; i < n; i += gridDim.x) {
      const int64_t from = a.long_list[i];
      const unsigned key = a.keys[(from + 1) * a.piece];  // the next piece's places are all the token's
      int64_t lo = from + 2, hi = a.pieces;               // first piece that does not begin with it: 64 places are looked at at a time
      while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const int with = __popcll(__ballot(at < hi && a.keys[at * a.piece] == key));
        if (with == 0) break;
        const int64_t known = lo + (with - 1) * step + 1;  // the last that has it is before this one
        hi = known + step - 1 < hi ? known + step - 1 : hi;
        lo = known;
      }
      const int64_t parts = lo - (from + 2), each = (parts + 7) / 8, b = wave * each, e = b + each < parts ? b + each : parts;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
      auto add = [&](const float* p) {
        if (left == 4) {
          sum += *reinterpret_cast<const f32x4_any*>(p);
          return;
        }
        for (int k = 0; k < left; ++k) sum[k] += p[k];
      };
      if (left > 0) {
        if (wave == 0) add(a.partial + (from * 2 + 1) * a.channels + c);
#pragma unroll 4
        for (int64_t x = b; x < e; ++x) add(a.partial + (from + 2 + x) * 2 * a.channels + c);
      }
      sums[wave][lane] = sum;
      __syncthreads();
      if (wave == 0 && left > 0) {
#pragma unroll
        for (int k = 1; k < 8; ++k) sum += sums[k][lane];
        G* p = static_cast<G*>(a.dtable) + (int64_t)key * a.channels + c;
        for (int k = 0; k < left; ++k) {
          float v = sum[k] * a.scale;
          if (a.accumulate) v += (float)p[k];
          p[k] = (G)v;
        }
      }
      __syncthreads();
    }
  }
}

// ---- host -------------------------------------------------------------------------------------------------------------------
struct EmbedShape {
  int64_t T, ld;
  int V, D;
};
int embed_shape(const jz_embed_desc* d, EmbedShape* s) {
  if (!d) return JZ_ERR_NULL;
  if (d->tokens < 0 || d->vocab <= 0 || d->channels <= 0 || d->dtype < JZ_F16 || d->dtype > JZ_F32 || d->out_dtype < JZ_F16 || d->out_dtype > JZ_F32 ||
      !(fabsf(d->scale) < INFINITY))
    return JZ_ERR_SHAPE;
  *s = {d->tokens, d->out_stride ? d->out_stride : d->channels, d->vocab, d->channels};
  if (s->ld < s->D) return JZ_ERR_SHAPE;
  if ((d->out_dtype != d->dtype && d->out_dtype != JZ_F32) || s->D > (1 << 24) || s->ld > (1 << 24) || s->T >= int64_t(1) << 31) return JZ_ERR_UNSUPPORTED;
  // tensors larger than any card's memory
  if (std::max(s->T * s->ld, (int64_t)s->V * s->D) > int64_t(1) << 38) return JZ_ERR_UNSUPPORTED;
  return JZ_OK;
}
size_t bytes_of(int dtype) { return dtype == JZ_F32 ? 4 : 2; }
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
size_t stream_bytes(const EmbedShape& s, int dtype) { return s.T ? ((size_t)(s.T - 1) * s.ld + s.D) * bytes_of(dtype) : 0; }

struct SumPlan {
  int piece, lanes, slices;
  int64_t pieces;
};
SumPlan sum_plan(const EmbedShape& s) {
  SumPlan p;
  p.piece = s.T >= 32768 ? 32 : s.T >= 4096 ? 16 : 8;
  p.pieces = (s.T + p.piece - 1) / p.piece;
  const int64_t vecs = (s.D + 7) / 8;
  p.lanes = 8;
  while (p.lanes < vecs && p.lanes < 256) p.lanes *= 2;
  p.slices = (int)((vecs + p.lanes - 1) / p.lanes);
  return p;
}

struct EmbedLayout {
  SortLayout sort;
  size_t used, counter, list, partial, total;
};
EmbedLayout embed_layout(const EmbedShape& s) {
  EmbedLayout L;
  L.sort = sort_layout(s.T, s.V);
  const SumPlan p = sum_plan(s);
  size_t o = L.sort.total;
  L.used = o;
  o = up256(o + (size_t)s.V);
  L.counter = o;
  o += 256;
  L.list = o;
  o = up256(o + (size_t)p.pieces * 4);
  L.partial = o;
  if (s.T > 2 * p.piece) o = up256(o + (size_t)p.pieces * 2 * s.D * 4);
  L.total = o;
  return L;
}

template <class T, class O>
void lookup(const LookupArgs& a, hipStream_t st) {
  const bool few = a.channels < 8, stream = !few && (size_t)a.tokens * a.channels * sizeof(O) >= STREAM_BYTES;
  const int64_t each = few ? 8 : lookup_each<T, O>(stream), vecs = a.tokens * ((a.channels + each - 1) / each), of = 256 * 32 / each;
  const unsigned grid = (unsigned)std::min<int64_t>((vecs + of - 1) / of, EMBED_GRID);
  if (few) embed_lookup<T, O, true, false><<<grid, 256, 0, st>>>(a);
  else if (stream) embed_lookup<T, O, false, true><<<grid, 256, 0, st>>>(a);
  else embed_lookup<T, O, false, false><<<grid, 256, 0, st>>>(a);
}

template <class O, class G, bool STREAM>
void sum_launch(const SumArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(a.sum_blocks + a.zero_blocks, int64_t(1) << 23);
  if (grid == 0) return;
  const bool lines = a.ld * sizeof(O) % 128 == 0 && reinterpret_cast<uintptr_t>(a.dout) % 128 == 0;
  if (lines && (sizeof(O) == 2 || a.slices == 1) && (size_t)a.tokens * a.channels * sizeof(O) >= STREAM_BYTES) embed_sum<O, G, STREAM, true><<<grid, 256, 0, st>>>(a);
  else embed_sum<O, G, STREAM, false><<<grid, 256, 0, st>>>(a);
}
template <class O, class G>
int sums(const SumArgs& a, hipStream_t st) {
  if (sizeof(G) == 2 && (size_t)a.vocab * a.channels * sizeof(G) >= STREAM_BYTES) sum_launch<O, G, sizeof(G) == 2>(a, st);
  else sum_launch<O, G, false>(a, st);
  if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  if (a.tokens > 2 * a.piece) {
    const dim3 join((unsigned)std::min<int64_t>(a.pieces, 64), (unsigned)std::min<int64_t>((a.channels + 255) / 256, 64));
    embed_join<G><<<join, 512, 0, st>>>(a);
  }
  return jz::launch_status();
}

}  // namespace

extern "C" int jz_embed_fwd(const jz_embed_desc* d, const int* ids, const void* table, void* out, void* hip_stream) {
  EmbedShape s;
  const int rc = embed_shape(d, &s);
  if (rc != JZ_OK) return rc;
  if (!table || (s.T && (!ids || !out))) return JZ_ERR_NULL;
  if (s.T == 0) return JZ_OK;
  if ((reinterpret_cast<uintptr_t>(ids) & 3) || !jz::aligned16(table) || !jz::aligned16(out)) return JZ_ERR_ALIGN;
  const size_t n = stream_bytes(s, d->out_dtype);
  if (jz::overlaps(out, n, table, (size_t)s.V * s.D * bytes_of(d->dtype)) || jz::overlaps(out, n, ids, (size_t)s.T * 4)) return JZ_ERR_ALIAS;
  const LookupArgs a = {ids, table, out, s.T, s.ld, s.V, s.D, d->scale};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (d->dtype == JZ_F32) lookup<float, float>(a, st);
  else if (d->dtype == JZ_F16) d->out_dtype == JZ_F32 ? lookup<_Float16, float>(a, st) : lookup<_Float16, _Float16>(a, st);
  else d->out_dtype == JZ_F32 ? lookup<__bf16, float>(a, st) : lookup<__bf16, __bf16>(a, st);
  return jz::launch_status();
}

extern "C" int jz_embed_bwd_workspace_bytes(const jz_embed_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  EmbedShape s;
  const int rc = embed_shape(d, &s);
  if (rc != JZ_OK) return rc;
  *bytes = embed_layout(s).total;
  return JZ_OK;
}

extern "C" int jz_embed_bwd(const jz_embed_desc* d, const int* ids, const void* dout, int accumulate, void* dtable, void* ws, size_t ws_bytes, void* hip_stream) {
  EmbedShape s;
  int rc = embed_shape(d, &s);
  if (rc != JZ_OK) return rc;
  if (!dtable || (s.T && (!ids || !dout))) return JZ_ERR_NULL;
  const EmbedLayout L = embed_layout(s);
  if (!ws || ws_bytes < L.total) return JZ_ERR_WORKSPACE;
  if ((reinterpret_cast<uintptr_t>(ids) & 3) || !jz::aligned16(dout) || !jz::aligned16(dtable) || !jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const size_t n = stream_bytes(s, d->out_dtype), t = (size_t)s.V * s.D * bytes_of(d->dtype);
  if (jz::overlaps(dtable, t, dout, n) || jz::overlaps(dtable, t, ids, (size_t)s.T * 4) || jz::overlaps(dtable, t, ws, ws_bytes) || jz::overlaps(ws, ws_bytes, dout, n) ||
      jz::overlaps(ws, ws_bytes, ids, (size_t)s.T * 4))
    return JZ_ERR_ALIAS;
  if (s.T == 0 && accumulate) return JZ_OK;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* const b = static_cast<char*>(ws);
  SumArgs a = {};
  a.used = reinterpret_cast<unsigned char*>(b + L.used);
  a.n_long = reinterpret_cast<unsigned*>(b + L.counter);
  a.long_list = reinterpret_cast<unsigned*>(b + L.list);
  a.partial = reinterpret_cast<float*>(b + L.partial);
  rc = sort_tokens(L.sort, ids, s.T, s.V, accumulate ? nullptr : reinterpret_cast<unsigned char*>(b + L.used), a.n_long, b, &a.keys, &a.pos, st);
  if (rc != JZ_OK) return rc;
  const SumPlan p = sum_plan(s);
  a.dout = dout;
  a.dtable = dtable;
  a.tokens = s.T;
  a.ld = s.ld;
  a.pieces = p.pieces;
  a.vocab = s.V;
  a.channels = s.D;
  a.piece = p.piece;
  a.lanes = p.lanes;
  a.slices = p.slices;
  a.accumulate = accumulate != 0;
  a.scale = d->scale;
  const int64_t per = 256 / p.lanes;
  a.sum_blocks = (p.pieces * p.slices + per - 1) / per;
  a.zero_blocks = accumulate ? 0 : ((int64_t)s.V * s.D + ZERO_EACH - 1) / ZERO_EACH;
  if (d->dtype == JZ_F32) return sums<float, float>(a, st);
  if (d->dtype == JZ_F16) return d->out_dtype == JZ_F32 ? sums<float, _Float16>(a, st) : sums<_Float16, _Float16>(a, st);
  return d->out_dtype == JZ_F32 ? sums<float, __bf16>(a, st) : sums<__bf16, __bf16>(a, st);
}
