// The norms before and after a residual block, fused with the block's gate and the residual sum (include/jz.h:
// jz_norm_residual_fwd, jz_norm_residual_bwd).
//
//   p = y rstd(y) w_post,   r' = a r + s gate p,   n = r' rstd(r') w_pre,   rstd(v) = 1 / sqrt(mean v^2 + eps)
//
// One pass over the rows each way: a row stays in the registers of the THREADS lanes that share it (NV vectors of eight elements each)
// from its first element's load to its results' stores, so what moves is every tensor once.  The kernels are bound by memory.
// Backward the sums over rows (dw_pre, dw_post, dgate) stay in registers over a slab of consecutive rows, go to the workspace once a slab and are
// added up in a second launch, in the order of the rows.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "jz_internal.h"

namespace {

#include "jz_vec.h"

struct NormArgs {
  int64_t rows, rows_per_group, slab;
  int C;
  float eps, res_scale, branch_scale, inv_c;
  const void *r, *y;
  const float *w_post, *gate, *w_pre;
  void *r_out, *n;
  float *rstd_post, *rstd_pre;
  // backward
  const void *dr_out, *dn;
  void *dr, *dy, *dw_post, *dgate, *dw_pre;
  float* part;  // [slabs][4][C]: dw_pre, dw_post, dgate of the group that began before the slab, of the one that goes on behind it
  int slabs;
};

// the sum over the lanes that share a row, in every one of them
template <int THREADS>
__device__ __forceinline__ float row_sum(float s, float* lds) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  if constexpr (THREADS > 64) {
    constexpr int W = THREADS / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    s = lds[0];
#pragma unroll
    for (int i = 1; i < W; ++i) s += lds[i];
  }
  return s;
}
__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ f32x8 splat8(float v) { return f32x8{v, v, v, v, v, v, v, v}; }

// element index of a lane's vector i, and how many of its eight elements the row has
#define JZ_AT(i) (((i) * THREADS + lane) * 8)

// ROWS rows at a time in a workgroup of ROWS * THREADS lanes (ROWS > 1 only where a wavefront has a row alone)
template <class T, class R, int THREADS, int NV>
__global__ __launch_bounds__(THREADS >= 256 ? THREADS : 256) void norm_fwd(NormArgs a) {
  constexpr int ROWS = THREADS >= 256 ? 1 : 256 / THREADS;
  __shared__ float lds[2][THREADS >= 256 ? THREADS / 64 : 1];
  const bool branch = a.y, post = a.w_post, with_gate = a.gate, pre = a.n;
  const int lane = threadIdx.x % THREADS;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  if (row >= a.rows) return;  // whole wavefronts; with one row a workgroup the grid ends with the rows
  const T* y = static_cast<const T*>(a.y) + row * a.C;
  const R* r = static_cast<const R*>(a.r) + row * a.C;
  typename Vec8<R>::V rv[NV];
  typename Vec8<T>::V yv[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int left = a.C - JZ_AT(i);
    rv[i] = {};
    if (left > 0) rv[i] = load8(r + JZ_AT(i), left);
    if (branch) {
      yv[i] = {};
      if (left > 0) yv[i] = load8(y + JZ_AT(i), left);
    }
  }
  f32x8 o[NV];
  if (branch) {
    float k1 = 1.f;
    if (post) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const f32x8 v = widen8<T>(yv[i]);
        s += sum8(v * v);
      }
      k1 = 1.f / sqrtf(row_sum<THREADS>(s, lds[0]) * a.inv_c + a.eps);
      if (lane == 0) a.rstd_post[row] = k1;
    }
    const float* gate = with_gate ? a.gate + row / a.rows_per_group * a.C : nullptr;
    k1 *= a.branch_scale;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = a.C - JZ_AT(i);
      f32x8 p = widen8<T>(yv[i]) * k1;
      if (left > 0) {
        if (post) p *= load8(a.w_post + JZ_AT(i), left);
        if (with_gate) p *= load8(gate + JZ_AT(i), left);
      }
      o[i] = widen8<R>(rv[i]) * a.res_scale + p;
      if (left > 0) store8(static_cast<R*>(a.r_out) + row * a.C + JZ_AT(i), narrow8<R>(o[i]), left);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = widen8<R>(rv[i]);
  }
  if (pre) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s += sum8(o[i] * o[i]);
    const float k2 = 1.f / sqrtf(row_sum<THREADS>(s, lds[1]) * a.inv_c + a.eps);
    if (lane == 0) a.rstd_pre[row] = k2;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = a.C - JZ_AT(i);
      if (left > 0) store8(static_cast<T*>(a.n) + row * a.C + JZ_AT(i), narrow8<T>(o[i] * k2 * load8(a.w_pre + JZ_AT(i), left)), left);
    }
  }
}

// One workgroup of THREADS lanes takes the rows of a slab one after the other.
template <class T, class R, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void norm_bwd(NormArgs a) {
  __shared__ float lds[4][THREADS / 64];
  const bool branch = a.dy, post = a.w_post, with_gate = a.gate, pre = a.dn;
  const int lane = threadIdx.x;
  const int64_t first = (int64_t)blockIdx.x * a.slab, last = first + a.slab < a.rows ? first + a.slab : a.rows;
  f32x8 sum_pre[NV], sum_post[NV], sum_gate[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    sum_pre[i] = sum_post[i] = sum_gate[i] = splat8(0.f);
  }
  float* const part = a.part + (size_t)blockIdx.x * 4 * a.C;
  int64_t group = with_gate ? first / a.rows_per_group : 0;
  for (int64_t row = first; row < last; ++row) {
    const int turn = (int)(row - first) & 1;  // two sets of LDS cells: a row's sums are read while the next one's are written
    const float k1 = post ? a.rstd_post[row] : 1.f, k2 = pre ? a.rstd_pre[row] : 0.f;
    typename Vec8<R>::V tv[NV], ov[NV];
    typename Vec8<T>::V dv[NV], yv[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = a.C - JZ_AT(i);
      tv[i] = {};
      ov[i] = {};
      dv[i] = {};
      yv[i] = {};
      if (left > 0) {
        const int64_t at = row * a.C + JZ_AT(i);
        if (a.dr_out) tv[i] = load8(static_cast<const R*>(a.dr_out) + at, left);
        if (pre) {
          ov[i] = load8(static_cast<const R*>(a.r_out) + at, left);
          dv[i] = load8(static_cast<const T*>(a.dn) + at, left);
        }
        if (post || with_gate) yv[i] = load8(static_cast<const T*>(a.y) + at, left);
      }
    }
    float c2 = 0.f;
    if (pre) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int left = a.C - JZ_AT(i);
        const f32x8 t = widen8<T>(dv[i]) * (widen8<R>(ov[i]) * k2);  // dn rhat
        sum_pre[i] += t;
        if (left > 0) c2 += sum8(t * load8(a.w_pre + JZ_AT(i), left));
      }
      c2 = row_sum<THREADS>(c2, lds[turn]) * a.inv_c;
    }
    f32x8 e[NV];
    float c1 = 0.f;
    const float* gate = with_gate ? a.gate + group * a.C : nullptr;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int left = a.C - JZ_AT(i);
      f32x8 total = widen8<R>(tv[i]);
      if (pre) {
        const f32x8 w = left > 0 ? f32x8(load8(a.w_pre + JZ_AT(i), left)) : splat8(0.f);
        total += (widen8<T>(dv[i]) * w - widen8<R>(ov[i]) * (k2 * c2)) * k2;
      }
      if (left > 0) store8(static_cast<R*>(a.dr) + row * a.C + JZ_AT(i), narrow8<R>(total * a.res_scale), left);
      if (branch) {
        f32x8 b = total * a.branch_scale, yh = widen8<T>(yv[i]) * k1;
        if (with_gate) {
          f32x8 q = yh * b;
          if (post)
            if (left > 0) q *= load8(a.w_post + JZ_AT(i), left);
          sum_gate[i] += q;
          if (left > 0) b *= load8(gate + JZ_AT(i), left);
        }
        if (post) {
          sum_post[i] += b * yh;
          if (left > 0) b *= load8(a.w_post + JZ_AT(i), left);
          c1 += sum8(b * yh);
        }
        e[i] = b;
      }
    }
    if (branch) {
      if (post) c1 = row_sum<THREADS>(c1, lds[2 + turn]) * a.inv_c;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int left = a.C - JZ_AT(i);
        f32x8 d = e[i];
        if (post) d = (d - widen8<T>(yv[i]) * (k1 * c1)) * k1;
        if (left > 0) store8(static_cast<T*>(a.dy) + row * a.C + JZ_AT(i), narrow8<T>(d), left);
      }
    }
    if (with_gate) {
      const int64_t begin = group * a.rows_per_group, end = begin + a.rows_per_group;
      if (row + 1 == end || row + 1 == last) {  // the group or the slab ends: whole groups are done, others go to the workspace
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int left = a.C - JZ_AT(i);
          if (left > 0) {
            if (begin >= first && end <= last) store8(static_cast<T*>(a.dgate) + group * a.C + JZ_AT(i), narrow8<T>(sum_gate[i]), left);
            else store8(part + (begin < first ? 2 : 3) * a.C + JZ_AT(i), typename Vec8<float>::V(sum_gate[i]), left);
          }
          sum_gate[i] = splat8(0.f);
        }
        if (row + 1 == end) ++group;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int left = a.C - JZ_AT(i);
    if (left <= 0) continue;
    if (pre) store8(part + JZ_AT(i), sum_pre[i], left);
    if (post) store8(part + a.C + JZ_AT(i), sum_post[i], left);
  }
}

// Adds the slabs' sums up in the order of the rows: 64 columns a workgroup, its four wavefronts take a quarter of the slabs each.
// blockIdx.y: 0 dw_pre, 1 dw_post, from 2 on the gate's groups that cross a slab's end, by group or, where those are more, by slab.
constexpr int JOIN_WAVES = 4;
template <class T>
__global__ __launch_bounds__(64 * JOIN_WAVES) void norm_join(NormArgs a, int64_t groups, int by_slab) {
  __shared__ float lds[JOIN_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane, what = blockIdx.y;
  int64_t from = 0, to = a.slabs;  // slabs; the first one's sum is in part 3 for a gate, the others' in part 2
  void* out = a.dw_pre;
  if (what == 0 && !a.dw_pre) return;
  if (what == 1) {
    if (!a.dw_post) return;
    out = a.dw_post;
  }
  int64_t group = 0;
  if (what >= 2) {
    if (!a.dgate) return;
    if (by_slab) {  // the group that begins in this slab and goes on behind it
      const int64_t s = what - 2, end = (s + 1) * a.slab;
      if (end >= a.rows) return;
      group = (end - 1) / a.rows_per_group;
      if (group * a.rows_per_group < s * a.slab || (group + 1) * a.rows_per_group <= end) return;
    } else {
      group = what - 2;
    }
    from = group * a.rows_per_group / a.slab;
    to = ((group + 1) * a.rows_per_group - 1) / a.slab + 1;
    if (a.rows > 0 && to - from == 1) return;  // whole inside one slab: written there
    if (a.rows == 0) to = from;
    out = static_cast<T*>(a.dgate) + group * a.C;
  }
  float s = 0.f;
  if (col < a.C) {
    const int64_t each = (to - from + JOIN_WAVES - 1) / JOIN_WAVES, lo = from + wave * each, hi = lo + each < to ? lo + each : to;
    for (int64_t k = lo; k < hi; ++k) s += a.part[((size_t)k * 4 + (what < 2 ? what : k == from ? 3 : 2)) * a.C + col];
  }
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < a.C) static_cast<T*>(out)[col] = (T)((lds[0][lane] + lds[1][lane]) + (lds[2][lane] + lds[3][lane]));
}

// ---- host ---------------------------------------------------------------------------------------------------------------
constexpr int NORM_MAX_C = 16384;
constexpr int NORM_SLABS = 512;  // at most

struct Tensor {
  const void* p;
  size_t bytes;
  bool out;
};
int look_over(const Tensor* t, int n, const void* ws, size_t ws_bytes) {
  for (int i = 0; i < n; ++i)
    if (t[i].p && !jz::aligned16(t[i].p)) return JZ_ERR_ALIGN;
  for (int i = 0; i < n; ++i) {
    if (jz::overlaps(t[i].p, t[i].bytes, ws, ws_bytes)) return JZ_ERR_ALIAS;
    for (int j = i + 1; j < n; ++j)
      if ((t[i].out || t[j].out) && jz::overlaps(t[i].p, t[i].bytes, t[j].p, t[j].bytes)) return JZ_ERR_ALIAS;
  }
  return JZ_OK;
}

int norm_shape(const jz_norm_residual_desc* d, int64_t* groups, int64_t* per) {
  if (!d) return JZ_ERR_NULL;
  if (d->rows < 0 || d->channels <= 0 || d->rows_per_group < 0 || d->dtype < JZ_F16 || d->dtype > JZ_F32) return JZ_ERR_SHAPE;
  if (d->res_dtype != d->dtype && d->res_dtype != JZ_F32) return d->res_dtype < JZ_F16 || d->res_dtype > JZ_F32 ? JZ_ERR_SHAPE : JZ_ERR_UNSUPPORTED;
  if (!(d->eps >= 0.f && d->eps < INFINITY) || !(fabsf(d->res_scale) < INFINITY) || !(fabsf(d->branch_scale) < INFINITY)) return JZ_ERR_SHAPE;
  if (d->channels > NORM_MAX_C || d->rows > (int64_t(1) << 31) - 256) return JZ_ERR_UNSUPPORTED;
  *per = d->rows_per_group ? d->rows_per_group : std::max<int64_t>(d->rows, 1);
  if (d->rows % *per) return JZ_ERR_SHAPE;
  *groups = d->rows_per_group ? d->rows / *per : 1;
  return JZ_OK;
}
// A slab's sums are 16 bytes a channel; slabs of at least 8 rows, so that they are a small part of what moves.
int64_t slab_rows(int64_t rows) { return std::max<int64_t>(8, (rows + NORM_SLABS - 1) / NORM_SLABS); }
int slab_count(int64_t rows) { return (int)((rows + slab_rows(rows) - 1) / slab_rows(rows)); }

NormArgs norm_args(const jz_norm_residual_desc* d, int64_t per) {
  NormArgs a = {};
  a.rows = d->rows;
  a.rows_per_group = per;
  a.C = d->channels;
  a.eps = d->eps;
  a.res_scale = d->res_scale;
  a.branch_scale = d->branch_scale;
  a.inv_c = 1.f / (float)d->channels;
  return a;
}

// f(element type, residual type) for the descriptor's types
template <class F>
void with_types(const jz_norm_residual_desc* d, F&& f) {
  const bool wide = d->res_dtype == JZ_F32;
  if (d->dtype == JZ_F32) f(float(), float());
  else if (d->dtype == JZ_F16) wide ? f(_Float16(), float()) : f(_Float16(), _Float16());
  else wide ? f(__bf16(), float()) : f(__bf16(), __bf16());
}
template <int N>
using Int = std::integral_constant<int, N>;
// Lanes that share a row, and vectors of eight elements a lane: a wavefront alone up to 1024 channels (no barrier), more lanes
// above, so that a lane keeps at most 16 elements of every tensor in registers.
template <class F>
void with_lanes(int channels, F&& f) {
  if (channels <= 512) f(Int<64>(), Int<1>());
  else if (channels <= 1024) f(Int<64>(), Int<2>());
  else if (channels <= 2048) f(Int<256>(), Int<1>());
  else if (channels <= 4096) f(Int<256>(), Int<2>());
  else if (channels <= 8192) f(Int<512>(), Int<2>());
  else f(Int<1024>(), Int<2>());
}

}  // namespace

extern "C" int jz_norm_residual_fwd(const jz_norm_residual_desc* d, const void* r, const void* y, const float* w_post, const float* gate,
                                    const float* w_pre, void* r_out, void* n, float* rstd_post, float* rstd_pre, void* hip_stream) {
  int64_t groups, per;
  const int rc = norm_shape(d, &groups, &per);
  if (rc != JZ_OK) return rc;
  const bool branch = r_out != nullptr, post = w_post != nullptr, pre = n != nullptr;
  if (d->rows == 0) return JZ_OK;
  if (!r || (branch && !y) || (!branch && !pre) || (post && (!branch || !rstd_post)) || (gate && !branch) || (pre && (!w_pre || !rstd_pre))) return JZ_ERR_NULL;
  const size_t e = (size_t)d->rows * d->channels, tb = d->dtype == JZ_F32 ? 4 : 2, rb = d->res_dtype == JZ_F32 ? 4 : 2, c4 = (size_t)d->channels * 4;
  // r_out may be r: a row is in registers before its results are written
  const Tensor t[] = {{r == r_out ? nullptr : r, e * rb, false}, {branch ? y : nullptr, e * tb, false}, {w_post, c4, false}, {gate, c4 * groups, false}, {pre ? w_pre : nullptr, c4, false},
                      {r_out, e * rb, true}, {n, e * tb, true}, {post ? rstd_post : nullptr, (size_t)d->rows * 4, true}, {pre ? rstd_pre : nullptr, (size_t)d->rows * 4, true}};
  const int ok = look_over(t, 9, nullptr, 0);
  if (ok != JZ_OK) return ok;
  NormArgs a = norm_args(d, per);
  a.r = r; a.y = branch ? y : nullptr; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre;
  a.r_out = r_out; a.n = n; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  with_types(d, [&](auto te, auto re) {
    with_lanes(d->channels, [&](auto th, auto nv) {
      constexpr int TH = decltype(th)::value, ROWS = TH >= 256 ? 1 : 256 / TH;
      norm_fwd<decltype(te), decltype(re), TH, decltype(nv)::value><<<(unsigned)((a.rows + ROWS - 1) / ROWS), TH >= 256 ? TH : 256, 0, st>>>(a);
    });
  });
  return jz::launch_status();
}

extern "C" int jz_norm_residual_bwd_workspace_bytes(const jz_norm_residual_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  int64_t groups, per;
  const int rc = norm_shape(d, &groups, &per);
  if (rc == JZ_OK) *bytes = (size_t)slab_count(d->rows) * 4 * d->channels * sizeof(float);
  return rc;
}

extern "C" int jz_norm_residual_bwd(const jz_norm_residual_desc* d, const void* y, const void* r_out, const float* w_post, const float* gate,
                                    const float* w_pre, const float* rstd_post, const float* rstd_pre, const void* dr_out, const void* dn, void* dr,
                                    void* dy, void* dw_post, void* dgate, void* dw_pre, void* ws, size_t ws_bytes, void* hip_stream) {
  int64_t groups, per;
  const int rc = norm_shape(d, &groups, &per);
  if (rc != JZ_OK) return rc;
  const bool rows = d->rows > 0, branch = dy != nullptr, post = w_post != nullptr, pre = rows ? dn != nullptr : dw_pre != nullptr;
  if ((post && !dw_post) || (gate && !dgate) || (pre && (!dw_pre || !w_pre))) return JZ_ERR_NULL;
  if (rows && (!dr || (!pre && !dr_out) || ((post || gate) && !branch) || (branch && (post || gate) && !y) || (!branch && !pre) || (post && !rstd_post) || (pre && (!r_out || !rstd_pre))))
    return JZ_ERR_NULL;
  const size_t need = (size_t)slab_count(d->rows) * 4 * d->channels * sizeof(float);
  if (need && (!ws || ws_bytes < need)) return JZ_ERR_WORKSPACE;
  if (need && !jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const size_t e = (size_t)d->rows * d->channels, tb = d->dtype == JZ_F32 ? 4 : 2, rb = d->res_dtype == JZ_F32 ? 4 : 2, c4 = (size_t)d->channels * 4;
  const size_t r4 = (size_t)d->rows * 4, cb = (size_t)d->channels * tb;
  // dr may be dr_out
  const Tensor t[] = {{y, e * tb, false}, {pre ? r_out : nullptr, e * rb, false}, {w_post, c4, false}, {gate, c4 * groups, false}, {pre ? w_pre : nullptr, c4, false},
                      {post ? rstd_post : nullptr, r4, false}, {pre ? rstd_pre : nullptr, r4, false}, {dr_out == dr ? nullptr : dr_out, e * rb, false}, {dn, e * tb, false},
                      {dr, e * rb, true}, {dy, e * tb, true}, {post ? dw_post : nullptr, cb, true}, {gate ? dgate : nullptr, cb * groups, true}, {pre ? dw_pre : nullptr, cb, true}};
  const int ok = look_over(t, 14, ws, need);
  if (ok != JZ_OK) return ok;
  NormArgs a = norm_args(d, per);
  a.y = y; a.r_out = const_cast<void*>(r_out); a.w_post = w_post; a.gate = gate; a.w_pre = w_pre;
  a.rstd_post = const_cast<float*>(rstd_post); a.rstd_pre = const_cast<float*>(rstd_pre);
  a.dr_out = dr_out; a.dn = dn; a.dr = dr; a.dy = dy;
  a.dw_post = post ? dw_post : nullptr; a.dgate = gate ? dgate : nullptr; a.dw_pre = pre ? dw_pre : nullptr;
  a.part = static_cast<float*>(ws);
  a.slab = slab_rows(d->rows);
  a.slabs = slab_count(d->rows);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (rows) {
    with_types(d, [&](auto te, auto re) {
      with_lanes(d->channels, [&](auto th, auto nv) {
        norm_bwd<decltype(te), decltype(re), decltype(th)::value, decltype(nv)::value><<<(unsigned)a.slabs, decltype(th)::value, 0, st>>>(a);
      });
    });
    if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  }
  if (!a.dw_pre && !a.dw_post && !a.dgate) return JZ_OK;
  const int by_slab = a.slabs > 0 && groups > a.slabs;
  const dim3 grid((unsigned)((d->channels + 63) / 64), (unsigned)(2 + (a.dgate ? by_slab ? a.slabs : groups : 0)));
  with_types(d, [&](auto te, auto) { norm_join<decltype(te)><<<grid, 64 * JOIN_WAVES, 0, st>>>(a, groups, by_slab); });
  return jz::launch_status();
}
