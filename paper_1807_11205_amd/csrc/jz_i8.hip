// Products in 8-bit integers with a scale for each token and each channel (include/jz.h: jz_quantize_i8, jz_linear_i8, jz_ffn_i8_fwd).
//
//   scale = max |x| / 127 over a row,  q = x / scale to the nearest whole number (ties to even),   y[m][n] = RNE(sum over k of q_x q_w  *  s_x[m] s_w[n])
//
// The sums are int32 and exact, so no order or split of them matters.  Tokens get their codes in a launch of their own or, a few short
// ones, in every workgroup of the product.  The gated block's h is kept in FP32
// until it has codes: rounded to 16 bits first, one code in 700 (FP16) or in 90 (BF16) would be its neighbour, which an answer in FP16 shows.
//
// Bound: with few rows the weights' way from memory (jz_i8_few.h), with many the matrix instructions (jz_mm_tile.h), in between two launches that wait for each other (9 us).
// 16384 rows 4096 -> 12288 in BF16: 725 to 760 us, 50 of them codes (201 MB, 3.9 TB/s; a wavefront a row: a workgroup a row took 66).
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "jz_internal.h"

namespace {

#include "jz_lds_dma.h"
#include "jz_vec.h"
#include "jz_ffn_gemm.h"
#include "jz_mm_tile.h"

int64_t i8_pitch(int64_t cols) { return (cols + 15) & ~int64_t(15); }

// ---- codes --------------------------------------------------------------------------------------------------------------------
struct QuantArgs {
  const void* x;
  signed char* q;
  float* scale;
  int64_t rows, ld, pitch;
  int cols;
};
__device__ __forceinline__ unsigned magnitude8(f32x8 v) {  // NaN is larger than Inf, and Inf than every number
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ unsigned long long codes8(f32x8 v, float s, int left) {
  unsigned long long r = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float q = fminf(fmaxf(rintf(v[i] / s), -127.f), 127.f);  // (by 1 / s and a division near halves alone: the same time)
    r |= (unsigned long long)(unsigned char)(i < left ? (int)q : 0) << (8 * i);
  }
  return r;
}
// A row at a time by a wavefront (WIDE: by the workgroup); HOLD vectors of eight stay in a lane's registers, what is behind them is read twice.
template <class T, bool WIDE, int HOLD>
__global__ __launch_bounds__(256) void i8_quantize(QuantArgs a) {
  constexpr int LANES_ = WIDE ? 256 : 64;
  __shared__ unsigned most[4];
  const int t = WIDE ? threadIdx.x : threadIdx.x & 63;
  for (int64_t row = WIDE ? blockIdx.x : (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < a.rows; row += (int64_t)gridDim.x * (WIDE ? 1 : 4)) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ld;
    auto get = [&](int64_t c) { return c + 8 <= a.cols ? load8(x + c) : load8(x + c, c < a.cols ? (int)(a.cols - c) : 0); };
    typename Vec8<T>::V v[HOLD];
    unsigned m = 0;
#pragma unroll
    for (int j = 0; j < HOLD; ++j) v[j] = get(((int64_t)j * LANES_ + t) * 8);
#pragma unroll
    for (int j = 0; j < HOLD; ++j) m = max(m, magnitude8(widen8<T>(v[j])));
    for (int64_t c = ((int64_t)HOLD * LANES_ + t) * 8; c < a.cols; c += LANES_ * 8) m = max(m, magnitude8(widen8<T>(get(c))));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) m = max(m, (unsigned)__shfl_xor((int)m, d));
    if constexpr (WIDE) {
      if ((t & 63) == 0) most[t >> 6] = m;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 4; ++w) m = max(m, most[w]);
      __syncthreads();
    }
    const bool fine = m < 0x7f800000u;
    const float s = fine ? __uint_as_float(m) / 127.f : NAN;  // a row with Inf or NaN: every result of it is NaN
    if (t == 0) a.scale[row] = s;
    const bool none = !(s > 0.f);
    signed char* const q = a.q + row * a.pitch;
    auto put = [&](int64_t c, typename Vec8<T>::V w) {
      if (c < a.pitch) *reinterpret_cast<unsigned long long*>(q + c) = none ? 0ull : codes8(widen8<T>(w), s, c < a.cols ? (int)(a.cols - c) : 0);
    };
#pragma unroll
    for (int j = 0; j < HOLD; ++j) put(((int64_t)j * LANES_ + t) * 8, v[j]);
    for (int64_t c = ((int64_t)HOLD * LANES_ + t) * 8; c < a.pitch; c += LANES_ * 8) put(c, get(c));
  }
}
// A wavefront a row where it can hold it and there are rows for the whole chip, else a workgroup a row.
template <class T>
int quantize(const QuantArgs& a, hipStream_t st) {
  auto grid = [&](int64_t rows_each) { return (unsigned)std::min<int64_t>((a.rows + rows_each - 1) / rows_each, 1 << 20); };
  if (a.pitch <= 64 * 8 * 4) i8_quantize<T, false, 4><<<grid(4), 256, 0, st>>>(a);
  else if (a.pitch <= 64 * 8 * 8 && a.rows >= 1024) i8_quantize<T, false, 8><<<grid(4), 256, 0, st>>>(a);
  else i8_quantize<T, true, 4><<<grid(1), 256, 0, st>>>(a);
  return jz::launch_status();
}
int quantize(int dtype, const QuantArgs& a, hipStream_t st) {
  if (a.rows == 0) return JZ_OK;
  return dtype == JZ_F32 ? quantize<float>(a, st) : dtype == JZ_F16 ? quantize<_Float16>(a, st) : quantize<__bf16>(a, st);
}

#include "jz_i8_few.h"

// ---- products -----------------------------------------------------------------------------------------------------------------
struct I8Out {
  const float *sx, *sw, *su;  // scales of the tokens and of the channels (su: of the interleaved matrix)
  void* y;
  int64_t M, N, ld;
  int act;
};
// A lane has the same eight columns in every row that it stores; its scales are asked for together, from places that exist, before the first is needed.  (A load in each turn of the
// loop was waited for in each: 16384 rows, 4096 -> 12288, 778 us, so 764.)
template <class T>
struct I8Store : I8Out {
  bool stream;  // past the caches
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile&, int64_t m0, int64_t n0, int lane) const {
    constexpr int PER = S::COLS / 8, TURNS = PER / 2, EACH = 64 / PER;
    const int c = lane % PER * 8, row0 = lane / PER;
    const int64_t n = n0 + c;
    const int left = N - n < 8 ? (int)(N - n) : 8;
    float r[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) r[t] = sx[m0 + row0 + t * EACH < M ? m0 + row0 + t * EACH : M - 1];
    if (left <= 0) return;
    const f32x8 w = load8(sw + n, left);
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int row = row0 + t * EACH;
      const int64_t m = m0 + row;
      int v[8];
      s.row8(row, c, v);
      f32x8 f;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (float)v[e] * (r[t] * w[e]);
      if (m >= M) continue;
      T* const to = static_cast<T*>(y) + m * ld + n;
      if (stream && left == 8) stream8(to, narrow8<T>(f));
      else store8(to, narrow8<T>(f), left);
    }
  }
};
// gate and up alternate by 32 columns; h in FP32
struct I8Glu : I8Out {
  template <class S>
  __device__ __forceinline__ void strip(const S& s, const MmTile&, int64_t m0, int64_t n0, int lane) const {
    constexpr int PER = S::COLS / 16, TURNS = PER / 2, EACH = 64 / PER;
    const int c = lane % PER, from = (c >> 2) * 64 + (c & 3) * 8, row0 = lane / PER;
    const int64_t n = n0 / 2 + c * 8;
    const int left = N - n < 8 ? (int)(N - n) : 8;
    float r[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) r[t] = sx[m0 + row0 + t * EACH < M ? m0 + row0 + t * EACH : M - 1];
    if (left <= 0) return;
    const f32x8 wg = load8(sw + n, left), wu = load8(su + n, left);
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const int row = row0 + t * EACH;
      const int64_t m = m0 + row;
      int g[8], u[8];
      s.row8(row, from, g);
      s.row8(row, from + 32, u);
      f32x8 h;
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] = act_fwd(act, (float)g[e] * (r[t] * wg[e])) * ((float)u[e] * (r[t] * wu[e]));
      if (m < M) store8(static_cast<float*>(y) + m * ld + n, h, left);
    }
  }
};

MmArgs i8_args(const signed char* x, int64_t M, const void* w0, const void* w1, int64_t N, int64_t K) {
  MmArgs a = {};
  const int64_t pitch = i8_pitch(K);
  a.a = {{x, x}, M, pitch, 0};
  a.b = {{w0, w1 ? w1 : w0}, N, pitch, 0};
  a.row_bytes = pitch;
  return a;
}
// Fitted to 20 sizes from 128 x 1024 x 1024 to 5000 x 8000 x 5000, each with every tile; FP16, microseconds, without the quantising launch, 256 / 192 / 128 / 64: 4096^3 61 78 71 116,
// 1500 rows 4096 -> 6000 50 43 57 70, 3000 rows 2048 -> 3000 31 27 34 40, 2048 rows 4096 -> 4096 50 42 37 65, 1500^3 26 21 16 14; with that launch, the last 32, 512 rows 8192 -> 1024 87 - 54 32 43,
// 128 rows 1024 -> 1024 23 - 17 16 13.
constexpr MmTime I8_TIMES[] = {{256, 0., 10., 1.07, .75, 3.1e-3, 256, 1.},
                               {192, 0., 9.5, .84, .62, 1.7e-3, 256, .97},
                               {128, 7., 0., .64, .5, .95e-3, 512, .97},
                               {64, 6., 0., .34, 0., .88e-3, 256, .97},
                               {32, 5., 0., .2, 0., 1.1e-3, 256, .97}};
// Two products and the activation: 128 only where it is expected to take a seventh less (4096 rows 2048 -> 5632 and back, all of it: 204 us with 256, 231 with 128, which the model has 3 % ahead).
constexpr MmTime GLU_TIMES[] = {I8_TIMES[0], {128, 7., 0., .64, .5, .95e-3, 512, .86}};
template <class T>
int i8_product(const MmArgs& a, const I8Out& o, hipStream_t st) {
  I8Store<T> e;
  static_cast<I8Out&>(e) = o;
  // past the caches, where the operands stay, if rows are whole halves of lines: 16384 rows 4096 -> 12288 in BF16 754 us with ordinary stores and 729 so, 8000 rows 1024 -> 12000 160 and 142; but
  // 7000 rows 500 -> 11000 85 and 95, and FP32 rows are stored as two halves of every 32 bytes
  e.stream = sizeof(T) == 2 && o.ld % 32 == 0 && reinterpret_cast<uintptr_t>(o.y) % 64 == 0 && (size_t)o.M * o.N * sizeof(T) >= STREAM_BYTES;
  switch (mm_tile_for(I8_TIMES, o.M, o.N, false, 1, a.row_bytes)) {
    case 256: return mm_launch<ElemI8, I8Store<T>, 256, false>(a, e, o.M, o.N, 1, st);
    case 192: return mm_launch<ElemI8, I8Store<T>, 192, false>(a, e, o.M, o.N, 1, st);
    case 128: return mm_launch<ElemI8, I8Store<T>, 128, false>(a, e, o.M, o.N, 1, st);
    case 64: return mm_launch<ElemI8, I8Store<T>, 64, false>(a, e, o.M, o.N, 1, st);
  }
  return mm_launch<ElemI8, I8Store<T>, 32, false>(a, e, o.M, o.N, 1, st);
}
int i8_glu(const MmArgs& a, const I8Out& o, hipStream_t st) {
  I8Glu e;
  static_cast<I8Out&>(e) = o;
  const int64_t cols = (o.N + 31) / 32 * 64;
  if (mm_tile_for(GLU_TIMES, o.M, cols, false, 1, a.row_bytes) == 256) return mm_launch<ElemI8, I8Glu, 256, true>(a, e, o.M, cols, 1, st);
  return mm_launch<ElemI8, I8Glu, 128, true>(a, e, o.M, cols, 1, st);
}

// Few rows.  Codes of the tokens: from q and sx, or, where x is given, made in every workgroup.
constexpr int64_t FEW_TOKENS = 64;
bool few_quantize(int64_t M, int64_t K) { return M <= 4 && M * i8_pitch(K) <= FEW_CODES; }
template <class X, class Y, bool GLU, int TT, bool QUANTIZE>
int few_launch(const FewArgs& a, hipStream_t st) {
  // as many wavefronts as LDS holds, in one workgroup a compute unit or, where there are more of them, several
  constexpr int W = GLU && TT == 4 ? 4 : 8, CH = (TT == 1 || QUANTIZE) && !GLU ? 2 : 1;
  const unsigned grid = (unsigned)((a.N + 15) / 16);
  if (grid <= 256 || W == 4) i8_few<X, Y, GLU, TT, W, CH, QUANTIZE><<<grid, 64 * W, 0, st>>>(a);
  else i8_few<X, Y, GLU, TT, 4, CH, QUANTIZE><<<grid, 256, 0, st>>>(a);
  return jz::launch_status();
}
template <class X, class Y, bool GLU>
int few_product(const FewArgs& a, hipStream_t st) {
  if (a.x) return few_launch<X, Y, GLU, 1, true>(a, st);
  return a.M <= 16 ? few_launch<float, Y, GLU, 1, false>(a, st) : a.M <= 32 ? few_launch<float, Y, GLU, 2, false>(a, st) : few_launch<float, Y, GLU, 4, false>(a, st);
}

// ---- the calls ------------------------------------------------------------------------------------------------------------------
struct Rows {  // tokens as they come, and room for their codes
  const void* x;
  int dtype;
  int64_t M, K, ld;
  signed char* q;
  float* s;
};
template <class X, class Y>
int i8_run(const Rows& r, const void* w, const float* sw, void* y, int64_t N, int64_t ldy, hipStream_t st) {
  const bool in_place = few_quantize(r.M, r.K);
  if (!in_place) {
    const int rc = quantize(r.dtype, {r.x, r.q, r.s, r.M, r.ld, i8_pitch(r.K), (int)r.K}, st);
    if (rc != JZ_OK) return rc;
  }
  if (r.M <= FEW_TOKENS) {
    const signed char* c = static_cast<const signed char*>(w);
    return few_product<X, Y, false>({r.q, {c, c}, r.s, {sw, sw}, in_place ? r.x : nullptr, y, r.M, N, r.K, i8_pitch(r.K), r.ld, ldy, 0}, st);
  }
  return i8_product<Y>(i8_args(r.q, r.M, w, nullptr, N, r.K), {r.s, sw, nullptr, y, r.M, N, ldy, 0}, st);
}
template <class X>
int i8_run_glu(const Rows& r, const void* wg, const float* sg, const void* wu, const float* su, float* h, int64_t F, int act, hipStream_t st) {
  const bool in_place = few_quantize(r.M, r.K);
  if (!in_place) {
    const int rc = quantize(r.dtype, {r.x, r.q, r.s, r.M, r.ld, i8_pitch(r.K), (int)r.K}, st);
    if (rc != JZ_OK) return rc;
  }
  if (r.M <= FEW_TOKENS)
    return few_product<X, float, true>({r.q, {static_cast<const signed char*>(wg), static_cast<const signed char*>(wu)}, r.s, {sg, su}, in_place ? r.x : nullptr, h, r.M, F, r.K,
                                        i8_pitch(r.K), r.ld, F, act}, st);
  return i8_glu(i8_args(r.q, r.M, wg, wu, F, r.K), {r.s, sg, su, h, r.M, F, F, act}, st);
}

// ---- host -----------------------------------------------------------------------------------------------------------------------
struct I8Tensor {
  const void* p;
  size_t bytes, align;
  bool out;
};
int look_over(const I8Tensor* t, int n, const void* ws, size_t ws_bytes) {
  for (int i = 0; i < n; ++i)
    if (reinterpret_cast<uintptr_t>(t[i].p) & (t[i].align - 1)) return JZ_ERR_ALIGN;
  for (int i = 0; i < n; ++i) {
    if (jz::overlaps(t[i].p, t[i].bytes, ws, ws_bytes)) return JZ_ERR_ALIAS;
    for (int j = i + 1; j < n; ++j)
      if ((t[i].out || t[j].out) && jz::overlaps(t[i].p, t[i].bytes, t[j].p, t[j].bytes)) return JZ_ERR_ALIAS;
  }
  return JZ_OK;
}
size_t elem(int dtype) { return dtype == JZ_F32 ? 4 : 2; }
size_t span_of(int64_t rows, int64_t cols, int64_t ld, size_t each) { return rows ? ((size_t)(rows - 1) * ld + cols) * each : 0; }
size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

// the sums of K products of codes fit int32 up to here: 127^2 K < 2^31
constexpr int64_t I8_MOST = 131072;
constexpr int64_t I8_ROWS = int64_t(1) << 31, I8_ELEMENTS = int64_t(1) << 38;

struct I8Shape {
  int64_t M, K, N, ldx, ldy;
};
int i8_shape(const jz_linear_i8_desc* d, I8Shape* s) {
  if (!d) return JZ_ERR_NULL;
  if (d->rows < 0 || d->in_features <= 0 || d->out_features <= 0 || d->dtype < JZ_F16 || d->dtype > JZ_F32) return JZ_ERR_SHAPE;
  *s = {d->rows, d->in_features, d->out_features, d->x_stride ? d->x_stride : d->in_features, d->y_stride ? d->y_stride : d->out_features};
  if (s->ldx < s->K || s->ldy < s->N) return JZ_ERR_SHAPE;
  if (s->K > I8_MOST || s->N > (1 << 24) || std::max(s->ldx, s->ldy) > (1 << 24) || s->M > I8_ROWS) return JZ_ERR_UNSUPPORTED;
  if (std::max(s->M * std::max(s->ldx, s->ldy), s->N * s->K) > I8_ELEMENTS) return JZ_ERR_UNSUPPORTED;
  return JZ_OK;
}
struct I8Room {  // of M rows of codes
  size_t scales, total;
  I8Room(int64_t M, int64_t K) : scales(round256((size_t)M * i8_pitch(K))), total(scales + round256((size_t)M * 4)) {}
};
int ffn_i8_shape(const jz_ffn_desc* d, I8Shape* s, int64_t* F) {
  if (!d) return JZ_ERR_NULL;
  if (d->rows < 0 || d->in_features <= 0 || d->hidden <= 0 || d->out_features <= 0 || d->act < JZ_ACT_SILU || d->act > JZ_ACT_RELU || d->dtype < JZ_F16 || d->dtype > JZ_F32)
    return JZ_ERR_SHAPE;
  *s = {d->rows, d->in_features, d->out_features, d->x_stride ? d->x_stride : d->in_features, d->y_stride ? d->y_stride : d->out_features};
  *F = d->hidden;
  if (s->ldx < s->K || s->ldy < s->N) return JZ_ERR_SHAPE;
  if (d->dtype == JZ_F32 || s->K > I8_MOST || *F > I8_MOST || s->N > (1 << 24) || std::max(s->ldx, s->ldy) > (1 << 24) || s->M > I8_ROWS) return JZ_ERR_UNSUPPORTED;
  if (std::max(std::max(s->M * std::max(std::max(s->ldx, s->ldy), *F), s->N * *F), *F * s->K) > I8_ELEMENTS) return JZ_ERR_UNSUPPORTED;
  return JZ_OK;
}

}  // namespace

extern "C" int jz_quantize_i8(int64_t rows, int cols, int dtype, const void* x, int64_t x_stride, void* q, float* scale, void* hip_stream) {
  if (rows < 0 || cols <= 0 || dtype < JZ_F16 || dtype > JZ_F32) return JZ_ERR_SHAPE;
  const int64_t ld = x_stride ? x_stride : cols;
  if (ld < cols) return JZ_ERR_SHAPE;
  if (rows > I8_ROWS || ld > (1 << 24) || rows * ld > I8_ELEMENTS) return JZ_ERR_UNSUPPORTED;
  if (rows == 0) return JZ_OK;
  if (!x || !q || !scale) return JZ_ERR_NULL;
  const I8Tensor t[] = {{x, span_of(rows, cols, ld, elem(dtype)), 16, false}, {q, (size_t)rows * i8_pitch(cols), 16, true}, {scale, (size_t)rows * 4, 16, true}};
  const int rc = look_over(t, 3, nullptr, 0);
  if (rc != JZ_OK) return rc;
  return quantize(dtype, {x, static_cast<signed char*>(q), scale, rows, ld, i8_pitch(cols), cols}, static_cast<hipStream_t>(hip_stream));
}

extern "C" int jz_linear_i8_workspace_bytes(const jz_linear_i8_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  I8Shape s;
  const int rc = i8_shape(d, &s);
  if (rc != JZ_OK) return rc;
  *bytes = I8Room(s.M, s.K).total;
  return JZ_OK;
}

extern "C" int jz_linear_i8(const jz_linear_i8_desc* d, const void* x, const void* wq, const float* w_scale, void* y, void* ws, size_t ws_bytes, void* hip_stream) {
  I8Shape s;
  int rc = i8_shape(d, &s);
  if (rc != JZ_OK) return rc;
  if (!wq || !w_scale || (s.M && (!x || !y))) return JZ_ERR_NULL;
  if (s.M == 0) return JZ_OK;
  const I8Room room(s.M, s.K);
  if (!ws || ws_bytes < room.total) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const I8Tensor t[] = {{x, span_of(s.M, s.K, s.ldx, elem(d->dtype)), 16, false}, {wq, (size_t)s.N * i8_pitch(s.K), 16, false}, {w_scale, (size_t)s.N * 4, 16, false},
                        {y, span_of(s.M, s.N, s.ldy, elem(d->dtype)), 16, true}};
  rc = look_over(t, 4, ws, ws_bytes);
  if (rc != JZ_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  signed char* const q = static_cast<signed char*>(ws);
  const Rows r = {x, d->dtype, s.M, s.K, s.ldx, q, reinterpret_cast<float*>(q + room.scales)};
  if (d->dtype == JZ_F32) return i8_run<float, float>(r, wq, w_scale, y, s.N, s.ldy, st);
  if (d->dtype == JZ_F16) return i8_run<_Float16, _Float16>(r, wq, w_scale, y, s.N, s.ldy, st);
  return i8_run<__bf16, __bf16>(r, wq, w_scale, y, s.N, s.ldy, st);
}

extern "C" int jz_ffn_i8_workspace_bytes(const jz_ffn_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  I8Shape s;
  int64_t F;
  const int rc = ffn_i8_shape(d, &s, &F);
  if (rc != JZ_OK) return rc;
  *bytes = I8Room(s.M, s.K).total + I8Room(s.M, F).total + round256((size_t)s.M * F * 4);
  return JZ_OK;
}

extern "C" int jz_ffn_i8_fwd(const jz_ffn_desc* d, const void* x, const void* wq_gate, const float* s_gate, const void* wq_up, const float* s_up, const void* wq_down,
                             const float* s_down, void* y, void* ws, size_t ws_bytes, void* hip_stream) {
  I8Shape s;
  int64_t F;
  int rc = ffn_i8_shape(d, &s, &F);
  if (rc != JZ_OK) return rc;
  if (!wq_gate || !s_gate || !wq_up || !s_up || !wq_down || !s_down || (s.M && (!x || !y))) return JZ_ERR_NULL;
  if (s.M == 0) return JZ_OK;
  const I8Room rx(s.M, s.K), rh(s.M, F);
  if (!ws || ws_bytes < rx.total + rh.total + round256((size_t)s.M * F * 4)) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const size_t w = (size_t)F * i8_pitch(s.K), f = (size_t)F * 4;
  const I8Tensor t[] = {{x, span_of(s.M, s.K, s.ldx, 2), 16, false}, {wq_gate, w, 16, false}, {s_gate, f, 16, false}, {wq_up, w, 16, false}, {s_up, f, 16, false},
                        {wq_down, (size_t)s.N * i8_pitch(F), 16, false}, {s_down, (size_t)s.N * 4, 16, false}, {y, span_of(s.M, s.N, s.ldy, 2), 16, true}};
  rc = look_over(t, 8, ws, ws_bytes);
  if (rc != JZ_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* const b = static_cast<char*>(ws);
  signed char *const qx = reinterpret_cast<signed char*>(b), *const qh = qx + rx.total;
  float* const h = reinterpret_cast<float*>(b + rx.total + rh.total);
  const Rows tokens = {x, d->dtype, s.M, s.K, s.ldx, qx, reinterpret_cast<float*>(qx + rx.scales)}, hidden = {h, JZ_F32, s.M, F, F, qh, reinterpret_cast<float*>(qh + rh.scales)};
  if (d->dtype == JZ_F16) {
    rc = i8_run_glu<_Float16>(tokens, wq_gate, s_gate, wq_up, s_up, h, F, d->act, st);
    return rc == JZ_OK ? i8_run<float, _Float16>(hidden, wq_down, s_down, y, s.N, s.ldy, st) : rc;
  }
  rc = i8_run_glu<__bf16>(tokens, wq_gate, s_gate, wq_up, s_up, h, F, d->act, st);
  return rc == JZ_OK ? i8_run<float, __bf16>(hidden, wq_down, s_down, y, s.N, s.ldy, st) : rc;
}
