// Orthogonalised updates (include/jz.h: jz_orthogonalize, jz_muon_mp_update): Newton-Schulz products on the matrix instructions.
//
//   X = G / (||G|| + eps)  (transposed where G has more rows than columns: m <= n),   steps times   A = X X^T,  B = a I + b A + c A^2,  X <- B X
//
// Every step applies s -> a s + b s^3 + c s^5 to the singular values and leaves the singular vectors.  Small values grow by a (3.4) a step, and what is lost of them early
// grows with them; hence 22 bits an element, as two FP16 parts (jz_mm_tile.h), and FP32 sums.  Matrices are scaled by 2^11: values up to 31 are in FP16's range, and
// the low part of an element of 2^-12, the size that a normalised 4096 x 4096 matrix has, still has its bits.  A and B are symmetric: only tiles on and below the diagonal are
// computed, and stored twice.  X is kept in both orders, since it is an operand along both of its sides.
//
// Bound: the matrix instructions with large matrices (4096 x 12288, FP16 or BF16: 5.6 ms, 1.17 PFLOP/s of them; 16 of 2816 x 1024, the whole update: 2.2 ms, 0.2 of it memory's around the products), with
// small ones the launches, each of which waits for the one before (128 x 512: eight, 90 us; three of 1001 x 333, FP32: seventeen, 171 us).
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "jz_internal.h"

namespace {

#include "jz_lds_dma.h"
#include "jz_vec.h"
#include "jz_tile_schedule.h"
#include "jz_mm_tile.h"

constexpr float SCALE = 2048.f;
constexpr int PAD = 32;      // sides of the matrices in the workspace are multiples of this, zeros behind their ends

// workgroups that share a matrix's sum of squares
int sum_parts(int64_t elements, int64_t count) { return (int)std::max<int64_t>(1, std::min((elements + 8191) / 8192, std::max<int64_t>(1, 2048 / count))); }

// eight columns from col (a multiple of 8) on of a row of parts: 64 bytes of high parts of 32 columns, then their low parts
__device__ __forceinline__ void store_parts(char* row, int64_t col, const float (&v)[8]) {
  f16x8 hi, lo;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi[i] = (_Float16)v[i];
    lo[i] = (_Float16)(v[i] - (float)hi[i]);
  }
  char* const p = row + (col >> 5) * 128 + (col & 31) * 2;
  *reinterpret_cast<f16x8*>(p) = hi;
  *reinterpret_cast<f16x8*>(p + 64) = lo;
}
__device__ __forceinline__ void load_parts(const char* row, int64_t col, float (&v)[8]) {
  const char* const p = row + (col >> 5) * 128 + (col & 31) * 2;
  const f16x8 hi = *reinterpret_cast<const f16x8*>(p), lo = *reinterpret_cast<const f16x8*>(p + 64);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)hi[i] + (float)lo[i];
}

// ---- the matrix itself ----------------------------------------------------------------------------------------------------------
struct OrthoIn {
  const void* x;        // [count][rows][cols], stride elements apart: the matrix, or gradients
  float* momentum;      // of the update
  float inv_s, mu;
  const jz_loss_scale_state* state;
  int nesterov;
  int64_t count, rows, cols, stride;
  double *sums, *inv;   // [count][parts]; [count]
  int parts;
  float eps;
  const int* skip;
  int* found_inf;
};
// What is orthogonalised, eight elements from i on or the `left` that there are; v: the new momentum.
template <class T, bool MUON>
struct OrthoValue {
  const OrthoIn& a;
  float inv_s;
  __device__ __forceinline__ OrthoValue(const OrthoIn& a_) : a(a_), inv_s(MUON && a_.state ? 1.f / a_.state->scale : a_.inv_s) {}
  __device__ __forceinline__ f32x8 get(int64_t i, int left, f32x8* v) const {
    const f32x8 x = widen8<T>(load8(static_cast<const T*>(a.x) + i, left));
    if constexpr (!MUON) return x;
    const f32x8 g = x * inv_s;
    *v = a.mu * load8(a.momentum + i, left) + g;
    return a.nesterov ? g + a.mu * *v : *v;
  }
  // the squares of eight, NaN where a gradient is not finite; loads first, then what is made of them
  struct Raw {
    typename Vec8<T>::V x;
    f32x8 m;
  };
  __device__ __forceinline__ Raw ask(int64_t i) const {
    Raw r;
    r.x = load8(static_cast<const T*>(a.x) + i);
    if constexpr (MUON) r.m = load8(a.momentum + i);
    return r;
  }
  __device__ __forceinline__ double squares(const Raw& r) const {
    const f32x8 x = widen8<T>(r.x);
    double s = 0.;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float u = x[e];
      if constexpr (MUON) {
        const float g = x[e] * inv_s, v = a.mu * r.m[e] + g;
        u = a.nesterov ? g + a.mu * v : v;
      }
      s = fma((double)u, (double)u, s);
      if (MUON && !(fabsf(x[e]) < INFINITY)) s = NAN;
    }
    return s;
  }
};

// Partial sums of squares, in FP64; NaN where a gradient is not finite.  Memory: 16 x 2816 x 1024 gradients and momenta 68 us (4.1 TB/s).
template <class T, bool MUON>
__global__ __launch_bounds__(256) void ortho_sumsq(OrthoIn a) {
  constexpr int U = 4;  // groups of eight on their way at a time
  __shared__ double lds[4];
  const OrthoValue<T, MUON> in(a);
  const int64_t n = a.rows * a.cols, base = (int64_t)blockIdx.y * a.stride, step = (int64_t)a.parts * 2048;
  double s = 0.;
  int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  for (; i + (U - 1) * step + 8 <= n; i += U * step) {
    typename OrthoValue<T, MUON>::Raw r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = in.ask(base + i + u * step);
#pragma unroll
    for (int u = 0; u < U; ++u) s += in.squares(r[u]);
  }
  for (; i < n; i += step) {
    const int left = n - i < 8 ? (int)(n - i) : 8;
    typename OrthoValue<T, MUON>::Raw r = {};
    r.x = load8(static_cast<const T*>(a.x) + base + i, left);
    if (MUON) r.m = load8(a.momentum + base + i, left);
    s += in.squares(r);
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.sums[(int64_t)blockIdx.y * a.parts + blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__device__ __forceinline__ double ortho_factor(double s, float eps) {
  const double norm = sqrt(s) + (double)eps;
  return norm == 0. ? 0. : (double)SCALE / norm;
}
// Each matrix's factor; of the update, whether anything is to be done.  One workgroup, a wavefront a matrix.
template <bool MUON>
__global__ __launch_bounds__(1024) void ortho_factors(OrthoIn a) {
  __shared__ int bad;
  if (threadIdx.x == 0) bad = MUON && a.skip && *a.skip;
  __syncthreads();
  for (int64_t b = threadIdx.x >> 6; b < a.count; b += 16) {
    double s = 0.;
#pragma unroll 8
    for (int i = threadIdx.x & 63; i < a.parts; i += 64) s += a.sums[b * a.parts + i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) {
      a.inv[b] = ortho_factor(s, a.eps);
      if (MUON && !(s < INFINITY)) bad = 1;
    }
  }
  __syncthreads();
  if (MUON && threadIdx.x == 0) *a.found_inf = bad;
}

// The matrix in parts, in both orders: r [rows][cols], c [cols][rows].  A tile of 64 x 64 a workgroup.  Memory: as above 144 us for 830 MB.
struct OrthoParts {
  char *r, *c;
  int64_t rp, cp;  // padded sides
};
// FOLD: few sums, which every workgroup adds up by itself instead of a launch of one: 3 of 1001 x 333 161 and so 159 us, the update of 16 of 64 x 200 60.5 and 58.2.
constexpr int ORTHO_FOLD = 1024;
template <class T, bool MUON, bool FOLD>
__global__ __launch_bounds__(256) void ortho_parts(OrthoIn a, OrthoParts o) {
  __shared__ float tile[64][65];
  if (MUON && !FOLD && *a.found_inf) return;
  const OrthoValue<T, MUON> in(a);
  const int64_t across = (o.cp + 63) / 64, down = (o.rp + 63) / 64;
  const int64_t id = gridDim.x - 1 - blockIdx.x, of = id / (across * down), t = id - of * across * down;  // what was squared last is still in the last-level cache
  const int64_t r0 = t / across * 64, c0 = t % across * 64, base = of * a.stride;
  double inv;
  if constexpr (FOLD) {
    __shared__ double mine[4];
    __shared__ int bad[4];
    const int all = (int)a.count * a.parts, from = (int)of * a.parts;
    double s = 0.;
    bool wrong = MUON && a.skip && *a.skip;
    for (int i = threadIdx.x; i < a.parts; i += 256) s += a.sums[from + i];
    if (MUON)
      for (int i = threadIdx.x; i < all; i += 256) wrong |= !(a.sums[i] < INFINITY);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    wrong = __any(wrong);
    if ((threadIdx.x & 63) == 0) {
      mine[threadIdx.x >> 6] = s;
      bad[threadIdx.x >> 6] = wrong;
    }
    __syncthreads();
    inv = ortho_factor((mine[0] + mine[1]) + (mine[2] + mine[3]), a.eps);
    if (MUON) {
      wrong = bad[0] | bad[1] | bad[2] | bad[3];
      if (blockIdx.x == 0 && threadIdx.x == 0) *a.found_inf = wrong;
      if (wrong) return;
    }
  } else {
    inv = a.inv[of];
  }
  const int row = threadIdx.x / 8, col = threadIdx.x % 8 * 8;
#pragma unroll
  for (int h = 0; h < 64; h += 32) {
    const int64_t r = r0 + row + h, c = c0 + col;
    f32x8 u = {};
    if (r < a.rows && c < a.cols) {
      const int left = a.cols - c < 8 ? (int)(a.cols - c) : 8;
      const int64_t at = base + r * a.cols + c;
      f32x8 v;
      u = in.get(at, left, &v);
      if (MUON) store8(a.momentum + at, v, left);
#pragma unroll
      for (int e = 0; e < 8; ++e) u[e] = e < left ? (float)((double)u[e] * inv) : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[row + h][col + e] = u[e];
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < 64; h += 32) {
    float v[8];
    if (r0 + row + h < o.rp && c0 + col < o.cp) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile[row + h][col + e];
      store_parts(o.r + (of * o.rp + r0 + row + h) * o.cp * 4, c0 + col, v);
    }
    if (c0 + row + h < o.cp && r0 + col < o.rp) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile[col + e][row + h];
      store_parts(o.c + (of * o.cp + c0 + row + h) * o.rp * 4, r0 + col, v);
    }
  }
}

// ---- products -------------------------------------------------------------------------------------------------------------------
struct Parts {  // [matrix][rows][cols]
  char* p;
  int64_t rows, cols;
  __device__ __forceinline__ char* row(int64_t of, int64_t r) const { return p + (of * rows + r) * cols * 4; }
};
template <class S>
__device__ __forceinline__ void store_rows(const S& s, const Parts& to, int64_t of, int64_t m0, int64_t n0, int lane, float factor) {
  constexpr int PER = S::COLS / 8, EACH = 64 / PER;
  const int c = lane % PER * 8;
  char* const p = to.row(of, m0);
  if (n0 + c >= to.cols) return;
#pragma unroll
  for (int t = 0; t < 32 / EACH; ++t) {
    const int row = lane / PER + t * EACH;
    float v[8];
    s.row8(row, c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= factor;
    if (m0 + row < to.rows) store_parts(p + row * to.cols * 4, n0 + c, v);
  }
}
template <class S>
__device__ __forceinline__ void store_cols(const S& s, const Parts& to, int64_t of, int64_t m0, int64_t n0, int lane, float factor) {
  const int r = lane % 4 * 8;
  char* const p = to.row(of, n0);
  if (m0 + r >= to.cols) return;
#pragma unroll
  for (int t = 0; t < S::COLS / 16; ++t) {
    const int col = lane / 4 + t * 16;
    float v[8];
    s.col8(r, col, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= factor;
    if (n0 + col < to.rows) store_parts(p + col * to.cols * 4, m0 + r, v);
  }
}
struct OrthoSymmetric {  // a product that is its own transpose
  Parts a;
  float factor;
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile& w, int64_t m0, int64_t n0, int lane) const {
    store_rows(s, a, w.of, m0, n0, lane, factor);
    if (w.m != w.n) store_cols(s, a, w.of, m0, n0, lane, factor);
  }
};
struct OrthoSums {  // sums as they are, a tile on and one below the diagonal
  float* p;
  int64_t side;
  float factor;
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile& w, int64_t m0, int64_t n0, int lane) const {
    constexpr int PER = S::COLS / 8, EACH = 64 / PER;
    float* const to = p + w.of * side * side;
    float v[8];
    f32x8 f;
#pragma unroll
    for (int t = 0; t < 32 / EACH; ++t) {
      const int row = lane / PER + t * EACH, c = lane % PER * 8;
      s.row8(row, c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = v[e] * factor;
      if (m0 + row < side && n0 + c < side) store8(to + (m0 + row) * side + n0 + c, f);
    }
    if (w.m == w.n) return;
#pragma unroll
    for (int t = 0; t < S::COLS / 16; ++t) {
      const int col = lane / 4 + t * 16, r = lane % 4 * 8;
      s.col8(r, col, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = v[e] * factor;
      if (n0 + col < side && m0 + r < side) store8(to + (n0 + col) * side + m0 + r, f);
    }
  }
};
struct OrthoPoly {  // B = ca I + cb A + cc A^2
  Parts a, b;
  float ca, cb, cc;
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile& w, int64_t m0, int64_t n0, int lane) const {
    constexpr int PER = S::COLS / 8, EACH = 64 / PER, TURNS = 32 / EACH;
    const int c = lane % PER * 8, row0 = lane / PER;
    const int64_t n = n0 + c < a.cols ? n0 + c : 0;
    float u[TURNS][8];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) load_parts(a.row(w.of, m0 + row0 + t * EACH < a.rows ? m0 + row0 + t * EACH : 0), n, u[t]);  // together, before the first is needed
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int row = row0 + t * EACH;
      float v[8];
      s.row8(row, c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fmaf(cc / SCALE, v[e], fmaf(cb, u[t][e], m0 + row == n0 + c + e ? ca * SCALE : 0.f));
      s.set_row8(row, c, v);
      if (m0 + row < a.rows && n0 + c < a.cols) store_parts(b.row(w.of, m0 + row), n0 + c, v);
    }
    if (w.m != w.n) store_cols(s, b, w.of, m0, n0, lane, 1.f);
  }
};
struct OrthoApply {  // X <- B X
  Parts x, xt;
  float factor;
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile& w, int64_t m0, int64_t n0, int lane) const {
    store_rows(s, x, w.of, m0, n0, lane, factor);
    store_cols(s, xt, w.of, m0, n0, lane, factor);
  }
};
// The last B X: eight elements at a time to where they are stored, transposed back where TALL was transposed.
template <class Sink>
struct OrthoResult {
  Sink sink;
  int64_t m, n, stride;
  bool tall;
  float factor;
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile& w, int64_t m0, int64_t n0, int lane) const {
    constexpr int PER = S::COLS / 8, EACH = 64 / PER;
    float v[8];
    f32x8 f;
    if (!tall) {
      const int c = lane % PER * 8, left = n - n0 - c < 8 ? (int)(n - n0 - c) : 8;
      if (left <= 0) return;
#pragma unroll 2
      for (int t = 0; t < 32 / EACH; ++t) {
        const int row = lane / PER + t * EACH;
        s.row8(row, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v[e] * factor;
        if (m0 + row < m) sink.put(w.of * stride + (m0 + row) * n + n0 + c, f, left);
      }
    } else {
      const int r = lane % 4 * 8, left = m - m0 - r < 8 ? (int)(m - m0 - r) : 8;
      if (left <= 0) return;
#pragma unroll 2
      for (int t = 0; t < S::COLS / 16; ++t) {
        const int col = lane / 4 + t * 16;
        s.col8(r, col, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = v[e] * factor;
        if (n0 + col < n) sink.put(w.of * stride + (n0 + col) * m + m0 + r, f, left);
      }
    }
  }
};
// The result itself, rounded once.  (Operands rounded to FP16 in the last product of a BF16 result would save two thirds of it, 5.6 and 5.1 ms for 4096 x 12288, but P, up to 41 where X has
// little, would count their errors that many times: with a matrix of low rank 1 to 2 % of the result.)
template <class O>
struct OrthoStore {
  O* y;
  __device__ __forceinline__ void put(int64_t at, f32x8 v, int left) const { store8(y + at, narrow8<O>(v), left); }
};
// The update's master weights and their copy.
template <class T>
struct MuonStore {
  float* w;
  T* w16;
  float lr, update_scale, wd;
  __device__ __forceinline__ void put(int64_t at, f32x8 o, int left) const {
    const f32x8 v = load8(w + at, left);
    f32x8 r = v - lr * (update_scale * o + wd * v);
    lds_pin(r);  // rounded to FP32 here: the copy is that value's, and not the 16-bit rounding of a fused multiply-add
    store8(w + at, r, left);
    store8(w16 + at, narrow8<T>(r), left);
  }
};

#include "jz_ortho_chain.h"

// ---- host -------------------------------------------------------------------------------------------------------------------------
struct OrthoShape {
  int64_t count, rows, cols, stride, m, n, mp, np;
  bool tall;
};
int ortho_shape(const jz_ortho_desc* d, OrthoShape* s) {
  if (!d) return JZ_ERR_NULL;
  if (d->count < 0 || d->rows <= 0 || d->cols <= 0 || d->dtype < JZ_F16 || d->dtype > JZ_F32 || d->out_dtype < JZ_F16 || d->out_dtype > JZ_F32 || d->steps < 1 ||
      !(fabsf(d->a) < INFINITY) || !(fabsf(d->b) < INFINITY) || !(fabsf(d->c) < INFINITY) || !(d->eps >= 0.f && d->eps < INFINITY))
    return JZ_ERR_SHAPE;
  const int64_t each = (int64_t)d->rows * d->cols;
  *s = {d->count, d->rows, d->cols, d->stride ? d->stride : each, std::min(d->rows, d->cols), std::max(d->rows, d->cols), 0, 0, d->rows > d->cols};
  if (s->stride < each) return JZ_ERR_SHAPE;
  s->mp = (s->m + PAD - 1) / PAD * PAD;
  s->np = (s->n + PAD - 1) / PAD * PAD;
  if (s->n > (1 << 17) || d->steps > 64 || s->count > 65535 || s->stride > int64_t(1) << 35 || s->count * s->stride > int64_t(1) << 35 || s->count * s->mp * s->np > int64_t(1) << 35)
    return JZ_ERR_UNSUPPORTED;
  return JZ_OK;
}
size_t round256(size_t n) { return (n + 255) & ~size_t(255); }
struct OrthoLayout {
  size_t sums, inv, x, xt[2], a, b, more[4], total;
  bool short_side;
  OrthoLayout(const OrthoShape& s, const jz_ortho_desc* d);
};
template <class Epi>
int ortho_product(const Parts& p, const Parts& q, bool symmetric, int64_t count, const int* skip, const Epi& e, hipStream_t st) {
  MmArgs a = {};
  a.a = {{p.p, p.p}, p.rows, p.cols * 4, p.rows * p.cols * 4};
  a.b = {{q.p, q.p}, q.rows, q.cols * 4, q.rows * q.cols * 4};
  a.row_bytes = p.cols * 4;
  a.symmetric = symmetric;
  a.skip = skip;
  // Fitted to 25 sizes from 192 to 4096 squared (1 to 16 of them), each with every tile; FP16 inputs.  The model is within 10 % of most and its choice within 5 % of the best.  Smaller tiles
  // read the operands more often, which shows where they do not stay in the last-level cache (16 updates of 2816 x 1024: 2.14 ms with 256, 2.22 with the 128 that the model alone prefers for
  // K = 1024), hence the 7 %.  192 is there for what fills the chip with neither 256 nor 128: the symmetric product of 4096 x 4096 is 136 tiles of 256, 241 us, 253 of 192, 200 us, or 528 of
  // 128, 250 us; the whole of 4096 x 12288 in FP16 6.1 ms without it, 5.5 with.
  static constexpr MmTime kinds[] = {{256, 2., 12., 1.4, 1.1, 5.2e-3, 256, 1.},
                                     {192, 4., 12., .9, .66, 3.3e-3, 256, .93},
                                     {128, 6., 0., .68, .38, 1.55e-3, 256, .93},
                                     {64, 4.5, 0., .34, 0., 1.3e-3, 256, 1.},
                                     {32, 4., 0., .2, 0., 1.3e-3, 256, 1.}};
  const int64_t best = mm_tile_for(kinds, p.rows, q.rows, symmetric, count, a.row_bytes);
  if constexpr (!std::is_same<Epi, OrthoSums>::value) {  // those have 128 rows at most: as many tiles of 128, and each takes less
    if (best == 256) return mm_launch<ElemSplit, Epi, 256, false>(a, e, p.rows, q.rows, count, st);
    if (best == 192) return mm_launch<ElemSplit, Epi, 192, false>(a, e, p.rows, q.rows, count, st);
  }
  if (best == 128) return mm_launch<ElemSplit, Epi, 128, false>(a, e, p.rows, q.rows, count, st);
  if (best == 64) return mm_launch<ElemSplit, Epi, 64, false>(a, e, p.rows, q.rows, count, st);
  return mm_launch<ElemSplit, Epi, 32, false>(a, e, p.rows, q.rows, count, st);
}

// X X^T of a narrow X: as many workgroups to a tile as keep eight tiles of the sum (256 k) each and do not fill the chip.  Two phases of
// 64 x 4096: 109 us with one, 62 so; 16 of 2693 x 80: 128 and 109; with 128 and 640 workgroups in
// all instead of 256 131 and 115 (what the sums are read by is one workgroup), with 128 k and 512 k at least instead of 256 32 x 2000 takes 43, 47 and 43.
int gram_splits(const OrthoShape& s) {
  const int64_t tiles = s.mp / 32 * (s.mp / 32 + 1) / 2 * std::max<int64_t>(1, s.count);
  return (int)std::max<int64_t>(1, std::min(std::min<int64_t>(16, s.np / 256), 256 / tiles));
}
int ortho_gram_sums(const Parts& x, int64_t count, int splits, const int* skip, const OrthoSums& e, hipStream_t st) {
  if (splits == 1) return ortho_product(x, x, true, count, skip, e, st);
  MmArgs a = {};
  a.a = a.b = {{x.p, x.p}, x.rows, x.cols * 4, x.rows * x.cols * 4};
  a.row_bytes = x.cols * 4;
  a.symmetric = true;
  a.skip = skip;
  a.splits = splits;
  return mm_launch<ElemSplit, OrthoSums, 32, false>(a, e, x.rows, x.rows, count, st);
}

template <class T, bool MUON>
int ortho_norms(const OrthoIn& in, hipStream_t st) {
  ortho_sumsq<T, MUON><<<dim3((unsigned)in.parts, (unsigned)in.count), 256, 0, st>>>(in);
  return jz::launch_status();
}
template <class T, bool MUON>
int ortho_begin(const OrthoIn& in, const OrthoShape& s, const OrthoParts& o, hipStream_t st) {
  const int rc = ortho_norms<T, MUON>(in, st);
  if (rc != JZ_OK) return rc;
  const int64_t tiles = (o.rp + 63) / 64 * ((o.cp + 63) / 64) * s.count;
  if (s.count * in.parts <= ORTHO_FOLD) {
    ortho_parts<T, MUON, true><<<(unsigned)tiles, 256, 0, st>>>(in, o);
  } else {
    ortho_factors<MUON><<<1, 1024, 0, st>>>(in);
    ortho_parts<T, MUON, false><<<(unsigned)tiles, 256, 0, st>>>(in, o);
  }
  return jz::launch_status();
}

// Steps in the space of the shorter side.  With A = X X^T an iterate is P X, P a polynomial of A that commutes with it: while P and A are carried along (B of the step, P <- B P,
// A <- B A B: four symmetric m x m products a step), X itself is not needed.  But A has lost a value s of X that is below 2^-11 of the largest, s^2 being below FP32's last
// bit, so that X is made, and A from it, after three steps at most: by then A's error of 2^-24 has grown to some 2^-16 of the smallest values.  (Emulated in FP32 with 22-bit operands, five
// steps as 2 + 3, against 64 bits: 2.2e-6 to 4e-5 for spectra from flat to 1e-6, as the plain form's 2.4e-6 to 6e-5; five steps without X: 8e-5 to 3e-4.)
// Not for a result in FP32: in P the FP32 sums' errors of A grow with the square of what X's would, and where small values stand beside large ones that is more than FP32's own: normal
// elements, 64 x 64 6.4e-6 where the formulas in FP32 have 1.2e-6, 128 x 128 7.4e-6 and 1.4e-6, 1024 x 2816 5.4e-6 and 2.6e-6; with steps of X itself 0.9e-6, 0.9e-6 and 2.1e-6.  It costs 128 x 512
// 90 -> 113 us, 256 x 2048 153 -> 180, 4096 x 12288 5.8 -> 8.5 ms.  A result of 16 bits rounds 2e-4 of itself away or more, and an update's weights have O times lr.
int phases(int steps) { return (steps + 2) / 3; }
int first_phase(int steps) { return steps - 3 * (phases(steps) - 1); }
// multiply-adds, halves of symmetric products alone; a tenth less has to be saved at least.  Where a phase is one launch (jz_ortho_chain.h) there are fewer of those too.  Launches are not weighed: this
// way five steps are 18 products, with X itself 15, and by the tiles' model one matrix of 200 x 400 to 640 x 1000 takes 6 to 15 % longer this way (100 and 87 us, 181 and 167; the last one, measured in FP32, 198 and 187).
bool short_side(int steps, int64_t m, int64_t n) {
  if (m <= CHAIN_SIDE) return true;
  const double p = phases(steps), k = steps, r = (double)n / (double)m;
  return p * 3 * r + 4 * k - 3 * p < 0.9 * k * (3 * r + 1);
}

OrthoLayout::OrthoLayout(const OrthoShape& s, const jz_ortho_desc* d) : short_side(d->out_dtype != JZ_F32 && ::short_side(d->steps, s.m, s.n)) {
  size_t o = 0;
  auto room = [&](size_t bytes) {
    const size_t at = o;
    o += round256(bytes);
    return at;
  };
  const size_t wide = (size_t)s.count * s.mp * s.np * 4, square = (size_t)s.count * s.mp * s.mp * 4;
  sums = room(s.count ? (size_t)s.count * sum_parts(s.rows * s.cols, s.count) * 8 : 0);
  inv = room((size_t)s.count * 8);
  x = room(wide);
  xt[0] = room(wide);
  xt[1] = room(d->steps > 1 ? wide : 0);
  a = room(s.mp <= CHAIN_SIDE ? square * gram_splits(s) : square);
  b = room(square);
  for (int i = 0; i < 4; ++i) more[i] = room(short_side && (i > 1 || s.mp > CHAIN_SIDE) ? square : 0);  // narrow ones have A, A B in LDS
  total = o;
}

// steps of the phase that begins behind `done`
int phase_steps(const OrthoLayout& L, int steps, int done) { return !L.short_side ? 1 : done == 0 ? first_phase(steps) : 3; }

template <class Sink>
int ortho_steps(const jz_ortho_desc* d, const OrthoShape& s, const OrthoLayout& L, char* b, const Sink& sink, const int* skip, hipStream_t st) {
  auto square = [&](size_t at) { return Parts{b + at, s.mp, s.mp}; };
  const Parts x = {b + L.x, s.mp, s.np};
  Parts A = square(L.a), A1 = square(L.more[0]), C = square(L.more[1]), P = square(L.more[2]), P1 = square(L.more[3]);
  const Parts B = square(L.b);
  auto symmetric = [&](const Parts& p, const Parts& q, const Parts& to, float factor) { return ortho_product(p, q, true, s.count, skip, OrthoSymmetric{to, factor}, st); };
  // P grows to a^steps where X has nothing: each step that it takes up scales it down by the power of two from |a| on
  const float shrink = exp2f(-ceilf(log2f(std::max(1.f, fabsf(d->a)))));
  int turn = 0, rc = JZ_OK;
  for (int done = 0, steps; done < d->steps; done += steps) {
    steps = phase_steps(L, d->steps, done);
    const bool last = done + steps == d->steps;
    float small = 1.f;  // P in the workspace is SCALE small P
    if (s.mp <= CHAIN_SIDE) {
      for (int i = 1; i < steps; ++i) small *= shrink;
      float* const sums = reinterpret_cast<float*>(b + L.a);
      const int splits = gram_splits(s);
      rc = ortho_gram_sums(x, s.count, splits, skip, OrthoSums{sums, s.mp, 1.f / SCALE}, st);
      const ChainArgs chain = {sums, {steps > 1 ? P : B, P1}, splits, steps, d->a, d->b, d->c, shrink, skip};
      if (rc == JZ_OK) rc = ortho_chain_launch(chain, s.count, st);
      if ((steps - 1) & 1) std::swap(P, P1);
    } else {
      rc = symmetric(x, x, A, 1.f / SCALE);
      for (int i = 0; i < steps && rc == JZ_OK; ++i) {
        const Parts to = i == 0 && steps > 1 ? P : B;
        rc = ortho_product(A, A, true, s.count, skip, OrthoPoly{A, to, d->a, d->b, d->c}, st);
        if (rc == JZ_OK && i + 1 < steps) {
          rc = symmetric(to, A, C, 1.f / SCALE);
          if (rc == JZ_OK) rc = symmetric(C, to, A1, 1.f / SCALE);
          std::swap(A, A1);
        }
        if (rc == JZ_OK && i > 0) {
          rc = symmetric(B, P, P1, shrink / SCALE);
          small *= shrink;
          std::swap(P, P1);
        }
      }
    }
    if (rc != JZ_OK) return rc;
    const Parts xt = {b + L.xt[turn & 1], s.np, s.mp}, next = {b + L.xt[!(turn & 1)], s.np, s.mp};
    ++turn;
    const Parts by = steps > 1 ? P : B;
    if (!last) rc = ortho_product(by, xt, false, s.count, skip, OrthoApply{x, next, 1.f / (SCALE * small)}, st);
    else rc = ortho_product(by, xt, false, s.count, skip, OrthoResult<Sink>{sink, s.m, s.n, s.stride, s.tall, 1.f / (SCALE * SCALE * small)}, st);
    if (rc != JZ_OK) return rc;
  }
  return JZ_OK;
}
OrthoParts begin_parts(const OrthoShape& s, const OrthoLayout& L, char* b) {
  if (s.tall) return {b + L.xt[0], b + L.x, s.np, s.mp};
  return {b + L.x, b + L.xt[0], s.mp, s.np};
}
size_t bytes_of(int dtype) { return dtype == JZ_F32 ? 4 : 2; }
size_t batch_bytes(const OrthoShape& s, size_t each) { return s.count ? ((size_t)(s.count - 1) * s.stride + s.rows * s.cols) * each : 0; }

}  // namespace

extern "C" int jz_orthogonalize_workspace_bytes(const jz_ortho_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  OrthoShape s;
  const int rc = ortho_shape(d, &s);
  if (rc != JZ_OK) return rc;
  *bytes = s.count ? OrthoLayout(s, d).total : 0;
  return JZ_OK;
}

extern "C" int jz_orthogonalize(const jz_ortho_desc* d, const void* x, void* y, void* ws, size_t ws_bytes, void* hip_stream) {
  OrthoShape s;
  int rc = ortho_shape(d, &s);
  if (rc != JZ_OK) return rc;
  if (s.count == 0) return JZ_OK;
  if (!x || !y) return JZ_ERR_NULL;
  const OrthoLayout L(s, d);
  if (!ws || ws_bytes < L.total) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(x) || !jz::aligned16(y) || !jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const size_t nx = batch_bytes(s, bytes_of(d->dtype)), ny = batch_bytes(s, bytes_of(d->out_dtype));
  if (jz::overlaps(x, nx, y, ny) || jz::overlaps(x, nx, ws, ws_bytes) || jz::overlaps(y, ny, ws, ws_bytes)) return JZ_ERR_ALIAS;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* const b = static_cast<char*>(ws);
  OrthoIn in = {};
  in.x = x;
  in.count = s.count;
  in.rows = s.rows;
  in.cols = s.cols;
  in.stride = s.stride;
  in.sums = reinterpret_cast<double*>(b + L.sums);
  in.parts = s.count ? sum_parts(s.rows * s.cols, s.count) : 0;
  in.inv = reinterpret_cast<double*>(b + L.inv);
  in.eps = d->eps;
  const OrthoParts o = begin_parts(s, L, b);
  rc = d->dtype == JZ_F32 ? ortho_begin<float, false>(in, s, o, st) : d->dtype == JZ_F16 ? ortho_begin<_Float16, false>(in, s, o, st) : ortho_begin<__bf16, false>(in, s, o, st);
  if (rc != JZ_OK) return rc;
  if (d->out_dtype == JZ_F32) return ortho_steps(d, s, L, b, OrthoStore<float>{static_cast<float*>(y)}, nullptr, st);
  if (d->out_dtype == JZ_F16) return ortho_steps(d, s, L, b, OrthoStore<_Float16>{static_cast<_Float16*>(y)}, nullptr, st);
  return ortho_steps(d, s, L, b, OrthoStore<__bf16>{static_cast<__bf16*>(y)}, nullptr, st);
}

namespace {
int muon_shape(const jz_ortho_desc* d, OrthoShape* s) {
  const int rc = ortho_shape(d, s);
  if (rc != JZ_OK) return rc;
  if (d->dtype != d->out_dtype) return JZ_ERR_SHAPE;
  return d->dtype == JZ_F32 ? JZ_ERR_UNSUPPORTED : JZ_OK;
}
}  // namespace

extern "C" int jz_muon_mp_update_workspace_bytes(const jz_ortho_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  OrthoShape s;
  const int rc = muon_shape(d, &s);
  if (rc != JZ_OK) return rc;
  *bytes = OrthoLayout(s, d).total;
  return JZ_OK;
}

namespace {
// What an update reads before it writes anything: the checks that both calls share, and the arguments of the first launches.
int muon_in(const jz_ortho_desc* d, const jz_muon_hparams* hp, const jz_loss_scale_state* state_dev, const int* skip_dev, const float* momentum, const void* grad16, bool rest_there,
            int* found_inf_dev, void* ws, size_t ws_bytes, OrthoShape* s, OrthoIn* in) {
  const int rc = muon_shape(d, s);
  if (rc != JZ_OK) return rc;
  if (!hp || !found_inf_dev || (s->count && (!momentum || !grad16 || !rest_there))) return JZ_ERR_NULL;
  for (float v : {hp->lr, hp->momentum, hp->weight_decay, hp->update_scale})
    if (!(fabsf(v) < INFINITY)) return JZ_ERR_SHAPE;
  if (!state_dev && !(hp->loss_scale > 0.f && hp->loss_scale < 3.0e38f)) return JZ_ERR_SHAPE;
  const OrthoLayout L(*s, d);
  if (s->count && (!ws || ws_bytes < L.total)) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(momentum) || !jz::aligned16(grad16) || !jz::aligned16(ws) || (reinterpret_cast<uintptr_t>(found_inf_dev) & 3) || (reinterpret_cast<uintptr_t>(skip_dev) & 3) ||
      (reinterpret_cast<uintptr_t>(state_dev) & 7))
    return JZ_ERR_ALIGN;
  char* const b = static_cast<char*>(ws);
  *in = {};
  in->x = grad16;
  in->momentum = const_cast<float*>(momentum);
  in->inv_s = state_dev ? 1.f : 1.f / hp->loss_scale;
  in->mu = hp->momentum;
  in->state = state_dev;
  in->nesterov = hp->nesterov != 0;
  in->count = s->count;
  in->rows = s->rows;
  in->cols = s->cols;
  in->stride = s->stride;
  in->sums = reinterpret_cast<double*>(b + L.sums);
  in->parts = s->count ? sum_parts(s->rows * s->cols, s->count) : 0;
  in->inv = reinterpret_cast<double*>(b + L.inv);
  in->eps = d->eps;
  in->skip = skip_dev;
  in->found_inf = found_inf_dev;
  return JZ_OK;
}
struct Place {
  const void* p;
  size_t bytes;
};
// the first `written` of n places overlap nothing, and the workspace, the last of them, nothing either
bool apart(const Place* t, int written, int n) {
  for (int i = 0; i < n; ++i)
    for (int j = i + 1; j < n; ++j)
      if ((i < written || j == n - 1) && jz::overlaps(t[i].p, t[i].bytes, t[j].p, t[j].bytes)) return false;
  return true;
}
}  // namespace

extern "C" int jz_muon_mp_overflow(const jz_ortho_desc* d, const jz_muon_hparams* hp, const jz_loss_scale_state* state_dev, const int* skip_dev, const float* momentum, const void* grad16,
                                   int* found_inf_dev, void* ws, size_t ws_bytes, void* hip_stream) {
  OrthoShape s;
  OrthoIn in;
  const int rc = muon_in(d, hp, state_dev, skip_dev, momentum, grad16, true, found_inf_dev, ws, ws_bytes, &s, &in);
  if (rc != JZ_OK) return rc;
  const size_t n = batch_bytes(s, 1);
  const Place t[] = {{found_inf_dev, 4}, {momentum, 4 * n}, {grad16, 2 * n}, {skip_dev, 4}, {state_dev, sizeof(*state_dev)}, {ws, ws_bytes}};
  if (!apart(t, 1, 6)) return JZ_ERR_ALIAS;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.count) {
    const int launched = d->dtype == JZ_F16 ? ortho_norms<_Float16, true>(in, st) : ortho_norms<__bf16, true>(in, st);
    if (launched != JZ_OK) return launched;
  }
  ortho_factors<true><<<1, 1024, 0, st>>>(in);
  return jz::launch_status();
}

extern "C" int jz_muon_mp_update(const jz_ortho_desc* d, const jz_muon_hparams* hp, const jz_loss_scale_state* state_dev, const int* skip_dev, float* master_w, float* momentum,
                                 const void* grad16, void* weight16, int* found_inf_dev, void* ws, size_t ws_bytes, void* hip_stream) {
  OrthoShape s;
  OrthoIn in;
  int rc = muon_in(d, hp, state_dev, skip_dev, momentum, grad16, master_w && weight16, found_inf_dev, ws, ws_bytes, &s, &in);
  if (rc != JZ_OK) return rc;
  if (!jz::aligned16(master_w) || !jz::aligned16(weight16)) return JZ_ERR_ALIGN;
  const size_t n = batch_bytes(s, 1);
  const Place t[] = {{master_w, 4 * n}, {momentum, 4 * n}, {weight16, 2 * n}, {found_inf_dev, 4}, {grad16, 2 * n}, {skip_dev, 4}, {state_dev, sizeof(*state_dev)}, {ws, ws_bytes}};
  if (!apart(t, 4, 8)) return JZ_ERR_ALIAS;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (s.count == 0) {  // the flag alone
    ortho_factors<true><<<1, 1024, 0, st>>>(in);
    return jz::launch_status();
  }
  const OrthoLayout L(s, d);
  char* const b = static_cast<char*>(ws);
  const OrthoParts o = begin_parts(s, L, b);
  rc = d->dtype == JZ_F16 ? ortho_begin<_Float16, true>(in, s, o, st) : ortho_begin<__bf16, true>(in, s, o, st);
  if (rc != JZ_OK) return rc;
  if (d->dtype == JZ_F16) return ortho_steps(d, s, L, b, MuonStore<_Float16>{master_w, static_cast<_Float16*>(weight16), hp->lr, hp->update_scale, hp->weight_decay}, found_inf_dev, st);
  return ortho_steps(d, s, L, b, MuonStore<__bf16>{master_w, static_cast<__bf16*>(weight16), hp->lr, hp->update_scale, hp->weight_decay}, found_inf_dev, st);
}
