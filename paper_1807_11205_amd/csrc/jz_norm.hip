// The norms before and after a residual block, fused with the block's gate and the residual sum (include/jz.h:
// jz_norm_residual_fwd, jz_norm_residual_bwd).
//
//   p = y rstd(y) w_post,   r' = a r + s gate p,   n = r' rstd(r') w_pre,   rstd(v) = 1 / sqrt(mean v^2 + eps)
//
// One pass over the rows each way: a row stays in the registers of the THREADS lanes that share it (NV vectors of eight elements each)
// from its first element's load to its results' stores, so what moves is every tensor once.  The kernels are bound by memory: 16384 rows of
// 4096 channels, FP16 with an FP32 residual stream, forward 174 us and backward 218 with its second launch 6 (4.1 TB/s in all; a copy reaches 4.8 to 5.1).
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
  int64_t step;   // backward: from one of a slab's rows to the next
  int64_t first;  // forward: the launch's first row
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

// Which elements of a row a lane has: NV vectors of eight, vector i from element 8 (i THREADS + lane) on.  Loads are not predicated, so that all of a row's are on
// their way at once: a vector that would pass the row's end is the row's last eight elements instead, and what of it lies outside the lane's own part is left
// out of the sums.  What a lane then stores a second time are the bits that their owner stores, except where the call works in place and the owner is in another
// wavefront: the owner may not have loaded yet, or, where no barrier lies between a row's loads and its stores (forward without a post-norm), have stored already, so that
// all that this lane makes of those elements is wrong.  There a lane stores its own elements alone, of every result.  (Backward a barrier lies between: dr alone needs it.)
//   EVEN   channels are a multiple of 8: a vector is a lane's own or nobody's        RAGGED   others from 8 on: the last vector overlaps its neighbour
//   TINY   less than 8: one vector, element by element
#define JZ_GLOBAL __attribute__((address_space(1)))
enum { EVEN = 0, RAGGED = 1, TINY = 2 };
template <int MODE, int THREADS>
struct Lane {
  int C, lane;
  __device__ __forceinline__ int own(int i) const { return (i * THREADS + lane) * 8; }
  __device__ __forceinline__ int at(int i) const { return MODE == TINY || own(i) + 8 <= C ? own(i) : C - 8; }
  __device__ __forceinline__ bool on(int i) const { return own(i) < C; }
  template <class T>
  __device__ __forceinline__ typename Vec8<T>::V load(const T* row, int i) const {
    if constexpr (MODE == TINY) {
      typename Vec8<T>::V v = {};
      if (on(i)) v = load8(row + own(i), C - own(i));
      return v;
    } else {
      // one address a wavefront and 32-bit offsets a lane: registers are short backward
      const JZ_GLOBAL char* base = (const JZ_GLOBAL char*)row;
      return *reinterpret_cast<const JZ_GLOBAL typename Vec8<T>::U*>(base + (unsigned)at(i) * (unsigned)sizeof(T));
    }
  }
  template <class T>
  __device__ __forceinline__ void store(T* row, int i, f32x8 v, bool in_place = false) const {
    if (!on(i)) return;
    if constexpr (MODE == TINY) {
      store8(row + own(i), narrow8<T>(v), C - own(i));
    } else if (MODE == RAGGED && in_place && own(i) + 8 > C) {
      const typename Vec8<T>::V o = narrow8<T>(v);
      const int skip = own(i) - at(i);
#pragma unroll
      for (int e = 1; e < 8; ++e)
        if (e >= skip) row[at(i) + e] = o[e];
    } else {
      JZ_GLOBAL char* base = (JZ_GLOBAL char*)row;
      *reinterpret_cast<JZ_GLOBAL typename Vec8<T>::U*>(base + (unsigned)at(i) * (unsigned)sizeof(T)) = narrow8<T>(v);
    }
  }
  __device__ __forceinline__ float sum(f32x8 v, int i) const {
    if constexpr (MODE == RAGGED) {
      const int skip = on(i) ? own(i) - at(i) : 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < skip ? 0.f : v[e];
    }
    const float s = sum8(v);
    return MODE == EVEN && !on(i) ? 0.f : s;
  }
};

// ROWS rows at a time in a workgroup of ROWS * THREADS lanes (ROWS > 1 only where a wavefront has a row alone)
template <class T, class R, int MODE, int THREADS, int NV>
__global__ __launch_bounds__(THREADS >= 256 ? THREADS : 256) void norm_fwd(NormArgs a) {
  constexpr int ROWS = THREADS >= 256 ? 1 : 256 / THREADS;
  __shared__ float lds[2][THREADS >= 256 ? THREADS / 64 : 1];
  const bool branch = a.y, post = a.w_post, with_gate = a.gate, pre = a.n;
  const Lane<MODE, THREADS> l = {a.C, (int)threadIdx.x % THREADS};
  const int64_t row = a.first + (int64_t)blockIdx.x * ROWS + threadIdx.x / THREADS;
  if (row >= a.rows) return;  // whole wavefronts; with one row a workgroup the grid ends with the rows
  typename Vec8<R>::V rv[NV];
  typename Vec8<T>::V yv[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    rv[i] = l.load(static_cast<const R*>(a.r) + row * a.C, i);
    yv[i] = {};
    if (branch) yv[i] = l.load(static_cast<const T*>(a.y) + row * a.C, i);
  }
  f32x8 o[NV];
  if (branch) {
    float k1 = 1.f;
    f32x8 w[NV];  // what y is multiplied by besides rstd
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w[i] = splat8(a.branch_scale);
      if (post) w[i] *= l.load(a.w_post, i);
      if (with_gate) w[i] *= l.load(a.gate + row / a.rows_per_group * a.C, i);
    }
    if (post) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const f32x8 v = widen8<T>(yv[i]);
        s += l.sum(v * v, i);
      }
      k1 = 1.f / sqrtf(row_sum<THREADS>(s, lds[0]) * a.inv_c + a.eps);
      if (l.lane == 0) a.rstd_post[row] = k1;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      o[i] = widen8<R>(rv[i]) * a.res_scale + widen8<T>(yv[i]) * k1 * w[i];
      l.store(static_cast<R*>(a.r_out) + row * a.C, i, o[i], a.r_out == a.r);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = widen8<R>(rv[i]);
  }
  if (pre) {
    f32x8 w[NV];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w[i] = l.load(a.w_pre, i);
      s += l.sum(o[i] * o[i], i);
    }
    const float k2 = 1.f / sqrtf(row_sum<THREADS>(s, lds[1]) * a.inv_c + a.eps);
    if (l.lane == 0) a.rstd_pre[row] = k2;
#pragma unroll
    for (int i = 0; i < NV; ++i) l.store(static_cast<T*>(a.n) + row * a.C, i, o[i] * k2 * w[i], a.r_out == a.r);
  }
}

// One workgroup of THREADS lanes takes the rows of a slab one after the other, the next row's loads ahead of a row's arithmetic; parameters and the sums over
// rows stay in registers.  A row's two means need one meeting of its lanes, not two: with q = branch_scale gate w_post y^ and t = w_pre dn,
//   c2 = mean(t r^),   c1 = mean(q R) = mean(q (dr_out + rstd_pre t)) - c2 mean(q rstd_pre r^)
// HAS: which tensors the call has, where that is usual.  A load in a branch keeps the compiler from counting the loads on their way, and a row would wait for the next one's.
enum { ANY = 0, BLOCK = 1, SUM = 2 };  // BLOCK: dn, dr_out and y (a post-norm or a gate); SUM: dn and dr_out, y is not needed
template <class T, class R, int MODE, int THREADS, int NV, int HAS>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 4 : 2) void norm_bwd(NormArgs a) {
  constexpr int W = THREADS / 64;
  // 1024 lanes have 128 registers each: two of the three sums and of the three parameters lie in LDS, every lane's in its own place, and no row is asked for
  // ahead; above 8192 channels, where LDS is full, the parameters are read for every row, and 48 to 91 registers are spilled all the same.  FP16 with an FP32 stream, both
  // launches: 8192 rows of 8192 channels 234 us, as fast as 512 lanes are (16384 of 4096: 224); 4096 rows of 16384, as many bytes, 550.
  constexpr bool WIDE = THREADS == 1024, REREAD = WIDE && NV > 1, KEPT = WIDE && !REREAD;
  __shared__ float lds[2][3][W];
  __shared__ f32x4 wide[WIDE ? (KEPT ? 4 : 2) * NV * 2 * THREADS : 1];
  const bool branch = HAS != ANY || a.dy, post = HAS != SUM && a.w_post, with_gate = HAS != SUM && a.gate, pre = HAS != ANY || a.dn, arrives = HAS != ANY || a.dr_out;
  const bool needs_y = HAS == BLOCK || (HAS == ANY && (post || with_gate));
  const Lane<MODE, THREADS> l = {a.C, (int)threadIdx.x};
  // Rows first, first + step, ...: with one gate for all the slabs are interleaved, since slabs of consecutive rows lie so far apart that workgroups side by side would
  // read the same few memory channels; with more, consecutive.
  const int64_t first = a.step == 1 ? blockIdx.x * a.slab : blockIdx.x, end_of_slab = a.step == 1 && first + a.slab < a.rows ? first + a.slab : a.rows;
  f32x8 sum_pre[NV], sum_post[WIDE ? 1 : NV], sum_gate[WIDE ? 1 : NV];
  auto from_lds = [&](int what, int i) {
    const f32x4* at = wide + ((what * NV + i) * 2) * THREADS + l.lane;
    const f32x4 lo = at[0], hi = at[THREADS];
    return f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  auto to_lds = [&](int what, int i, f32x8 v) {
    f32x4* at = wide + ((what * NV + i) * 2) * THREADS + l.lane;
    at[0] = f32x4{v[0], v[1], v[2], v[3]};
    at[THREADS] = f32x4{v[4], v[5], v[6], v[7]};
  };
  auto sum = [&](bool gate, int i) -> f32x8 {
    if constexpr (WIDE) return from_lds(gate, i);
    else return gate ? sum_gate[i] : sum_post[i];
  };
  auto put = [&](bool gate, int i, f32x8 v) {
    if constexpr (WIDE) to_lds(gate, i, v);
    else if (gate) sum_gate[i] = v;
    else sum_post[i] = v;
  };
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    sum_pre[i] = splat8(0.f);
    put(false, i, splat8(0.f));
    put(true, i, splat8(0.f));
  }
  float* const part = a.part + (size_t)blockIdx.x * 4 * a.C;
  int64_t group = with_gate ? first / a.rows_per_group : 0;

  struct Row {
    typename Vec8<R>::V t[NV], o[NV];
    typename Vec8<T>::V d[NV], y[NV];
    float k1, k2;
  } next, now;
  auto ask = [&](Row& v, int64_t row) {
    if constexpr (HAS == ANY) v.k1 = post ? a.rstd_post[row] : 1.f;
    else v.k1 = *(post ? a.rstd_post + row : a.rstd_pre + row);  // read and put away without a post-norm
    v.k2 = pre ? a.rstd_pre[row] : 0.f;
    const int64_t at = row * a.C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v.t[i] = v.o[i] = {};
      v.d[i] = v.y[i] = {};
      if (arrives) v.t[i] = l.load(static_cast<const R*>(a.dr_out) + at, i);
      if (pre) {
        v.o[i] = l.load(static_cast<const R*>(a.r_out) + at, i);
        v.d[i] = l.load(static_cast<const T*>(a.dn) + at, i);
      }
      if (needs_y) v.y[i] = l.load(static_cast<const T*>(a.y) + at, i);
    }
  };
  f32x8 w_pre[REREAD ? 1 : NV], w_post[WIDE ? 1 : NV], w_gate[WIDE ? 1 : NV];
  auto parameter = [&](const float* from, int i) -> f32x8 { return from ? f32x8(l.load(from, i)) : splat8(1.f); };
  auto gate_row = [&](int i) -> f32x8 { return parameter(with_gate ? a.gate + group * a.C : nullptr, i) * a.branch_scale; };
  auto pre_of = [&](int i) -> f32x8 { return REREAD ? parameter(pre ? a.w_pre : nullptr, i) : w_pre[REREAD ? 0 : i]; };
  auto post_of = [&](int i) -> f32x8 { return REREAD ? parameter(a.w_post, i) : KEPT ? from_lds(2, i) : w_post[WIDE ? 0 : i]; };
  auto gate_of = [&](int i) -> f32x8 { return REREAD ? gate_row(i) : KEPT ? from_lds(3, i) : w_gate[WIDE ? 0 : i]; };
  auto keep_gate = [&](int i) {
    if constexpr (KEPT) to_lds(3, i, gate_row(i));
    else if constexpr (!REREAD) w_gate[i] = gate_row(i);
  };
  if (!REREAD && first < end_of_slab) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      w_pre[REREAD ? 0 : i] = parameter(pre ? a.w_pre : nullptr, i);
      if constexpr (KEPT) to_lds(2, i, parameter(a.w_post, i));
      else w_post[WIDE ? 0 : i] = parameter(a.w_post, i);
      keep_gate(i);
    }
  }
  if (!WIDE && first < end_of_slab) ask(next, first);
  int turn = 0;
  for (int64_t row = first; row < end_of_slab; row += a.step, turn ^= 1) {
    const bool last = row + a.step >= end_of_slab;
    if constexpr (WIDE) {
      ask(now, row);
    } else {
      now = next;
      ask(next, last ? row : row + a.step);
    }
    const float k1 = post ? now.k1 : 1.f, k2 = now.k2;
    float s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const f32x8 hat = widen8<R>(now.o[i]) * k2, d = widen8<T>(now.d[i]);
      f32x8 t = splat8(0.f);
      if (pre) {
        sum_pre[i] += d * hat;
        t = d * pre_of(i);
        s1 += l.sum(t * hat, i);
      }
      if (post) {
        const f32x8 u = gate_of(i) * post_of(i) * (widen8<T>(now.y[i]) * k1);
        s2 += l.sum(u * (widen8<R>(now.t[i]) + t * k2), i);
        s3 += l.sum(u * hat, i);
      }
    }
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) {
      s1 += __shfl_xor(s1, m);
      s2 += __shfl_xor(s2, m);
      s3 += __shfl_xor(s3, m);
    }
    if constexpr (W > 1) {
      float(*cell)[W] = lds[turn];  // two sets: a row's sums are read while the next one's are written
      if ((l.lane & 63) == 0) {
        cell[0][l.lane >> 6] = s1;
        cell[1][l.lane >> 6] = s2;
        cell[2][l.lane >> 6] = s3;
      }
      // the wavefronts meet over LDS alone: the next row's loads stay on their way
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
      s1 = cell[0][0];
      s2 = cell[1][0];
      s3 = cell[2][0];
#pragma unroll
      for (int i = 1; i < W; ++i) {
        s1 += cell[0][i];
        s2 += cell[1][i];
        s3 += cell[2][i];
      }
    }
    const float c2 = s1 * a.inv_c, c1 = (s2 - c2 * (s3 * k2)) * a.inv_c;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int64_t at = row * a.C;
      const f32x8 hat = widen8<R>(now.o[i]) * k2, yh = widen8<T>(now.y[i]) * k1;
      f32x8 total = widen8<R>(now.t[i]);
      if (pre) total += (widen8<T>(now.d[i]) * pre_of(i) - hat * c2) * k2;
      l.store(static_cast<R*>(a.dr) + at, i, total * a.res_scale, a.dr == a.dr_out);
      if (branch) {
        if (with_gate) put(true, i, sum(true, i) + yh * post_of(i) * (total * a.branch_scale));
        f32x8 e = gate_of(i) * total;
        if (post) {
          put(false, i, sum(false, i) + e * yh);
          e = (e * post_of(i) - yh * c1) * k1;
        }
        l.store(static_cast<T*>(a.dy) + at, i, e);
      }
    }
    if (with_gate) {
      const int64_t begin = group * a.rows_per_group, end = begin + a.rows_per_group;
      if (row + 1 == end || last) {  // the group or the slab ends: whole groups are done, others go to the workspace
        const bool whole = a.step == 1 ? begin >= first && end <= end_of_slab : gridDim.x == 1, began = a.step == 1 ? begin < first : blockIdx.x > 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (whole) l.store(static_cast<T*>(a.dgate) + group * a.C, i, sum(true, i));
          else l.store(part + (began ? 2 : 3) * a.C, i, sum(true, i));
          put(true, i, splat8(0.f));
        }
        if (!last) {
          ++group;
#pragma unroll
          for (int i = 0; i < NV; ++i) keep_gate(i);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (pre) l.store(part, i, sum_pre[i]);
    if (post) l.store(part + a.C, i, sum(false, i));
  }
}

// Adds the slabs' sums up in the order of the rows: 64 columns a workgroup, its sixteen wavefronts take a sixteenth of the slabs each, eight
// loads at a time.
// blockIdx.y: 0 dw_pre, 1 dw_post, from 2 on the gate's groups that cross a slab's end, by group or, where those are more, by slab; short ones (alone) a
// wavefront each.
constexpr int JOIN_WAVES = 16;
template <class T>
__global__ __launch_bounds__(64 * JOIN_WAVES) void norm_join(NormArgs a, int64_t groups, int by_slab, int alone) {
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
    const int64_t number = alone ? (int64_t)(what - 2) * JOIN_WAVES + wave : what - 2;
    if (number >= (by_slab ? a.slabs : groups)) return;
    if (by_slab) {  // the group that begins in this slab and goes on behind it
      const int64_t s = number, end = (s + 1) * a.slab;
      if (end >= a.rows) return;
      group = (end - 1) / a.rows_per_group;
      if (group * a.rows_per_group < s * a.slab || (group + 1) * a.rows_per_group <= end) return;
    } else {
      group = number;
    }
    from = group * a.rows_per_group / a.slab;
    to = ((group + 1) * a.rows_per_group - 1) / a.slab + 1;
    if (a.rows > 0 && to - from == 1) return;  // whole inside one slab: written there
    if (a.rows == 0) to = from;
    out = static_cast<T*>(a.dgate) + group * a.C;
  }
  float s = 0.f;
  const bool whole = what >= 2 && alone;
  if (col < a.C) {
    const int64_t each = whole ? to - from : (to - from + JOIN_WAVES - 1) / JOIN_WAVES, lo = whole ? from : from + wave * each, hi = lo + each < to ? lo + each : to;
    const float* at = a.part + (what < 2 ? what : 2) * a.C + col;
    const size_t pitch = (size_t)4 * a.C;
    int64_t k = lo;
    if (what >= 2 && k == from && k < hi) s = at[k++ * pitch + a.C];
    for (; k + 8 <= hi; k += 8) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = at[(k + i) * pitch];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += v[i];
    }
    if (k < hi) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = at[(k + i < hi ? k + i : hi - 1) * pitch];
#pragma unroll
      for (int i = 0; i < 8; ++i) s += k + i < hi ? v[i] : 0.f;
    }
    if (whole) static_cast<T*>(out)[col] = (T)s;
  }
  if (whole) return;  // all of the workgroup's wavefronts
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < a.C) {
    s = lds[0][lane];
#pragma unroll
    for (int i = 1; i < JOIN_WAVES; ++i) s += lds[i][lane];
    static_cast<T*>(out)[col] = (T)s;
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
constexpr int NORM_MAX_C = 16384;
constexpr int NORM_SLABS = 512;  // half as many where a workgroup of the backward pass fills a compute unit

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
// A slab's sums are 16 bytes a channel, so slabs should be long, but a slab's rows follow one another, so they should be many.  At least four rows (BF16, both directions, at least
// eight: 1000 rows of 768 channels 20.8 us, four: 17.4; 333 rows of 4096: 30.1 and 20.3).  Up to 1024 channels, where a workgroup is one or two wavefronts, twice as many from
// 32 rows each on (65536 rows of 512 channels: 190 us with 512, 147 with 1024; 4096 rows of 1024 channels 30 and 34, which is why not below).
int64_t slab_rows(int64_t rows, int channels) {
  const int most = channels > 2048 ? NORM_SLABS / 2 : channels <= 1024 && rows >= 32 * NORM_SLABS ? 2 * NORM_SLABS : NORM_SLABS;
  return std::max<int64_t>(4, (rows + most - 1) / most);
}
int slab_count(int64_t rows, int channels) { return (int)((rows + slab_rows(rows, channels) - 1) / slab_rows(rows, channels)); }

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
// f(mode, lanes that share a row, vectors of eight elements a lane).  Forward a wavefront alone up to 1024 channels (no barrier), more lanes above, so that a lane
// keeps at most 16 elements of every tensor in registers.  Backward, where a lane also keeps parameters, their gradients and the next row, eight (up to 8192).
template <bool FORWARD, class F>
void with_lanes(int channels, F&& f) {
  auto sized = [&](auto mode) {
    if (channels <= 512) f(mode, Int<64>(), Int<1>());
    else if constexpr (FORWARD) {
      if (channels <= 1024) f(mode, Int<64>(), Int<2>());
      else if (channels <= 2048) f(mode, Int<256>(), Int<1>());
      else if (channels <= 4096) f(mode, Int<256>(), Int<2>());
      else if (channels <= 8192) f(mode, Int<512>(), Int<2>());
      else f(mode, Int<1024>(), Int<2>());
    } else {
      if (channels <= 1024) f(mode, Int<128>(), Int<1>());
      else if (channels <= 2048) f(mode, Int<256>(), Int<1>());
      else if (channels <= 4096) f(mode, Int<512>(), Int<1>());
      else if (channels <= 8192) f(mode, Int<1024>(), Int<1>());
      else f(mode, Int<1024>(), Int<2>());
    }
  };
  if (channels < 8) f(Int<TINY>(), Int<64>(), Int<1>());
  else if (channels % 8) sized(Int<RAGGED>());
  else sized(Int<EVEN>());
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
    with_lanes<true>(d->channels, [&](auto mode, auto th, auto nv) {
      constexpr int TH = decltype(th)::value, ROWS = TH >= 256 ? 1 : 256 / TH;
      constexpr int64_t LANES = TH >= 256 ? TH : 256, MOST = (int64_t(1) << 32) / LANES - 1;  // a launch has fewer than 2^32 lanes
      for (int64_t all = (a.rows + ROWS - 1) / ROWS, done = 0; done < all; done += MOST) {
        a.first = done * ROWS;
        norm_fwd<decltype(te), decltype(re), decltype(mode)::value, TH, decltype(nv)::value><<<(unsigned)std::min(all - done, MOST), (unsigned)LANES, 0, st>>>(a);
      }
    });
  });
  return jz::launch_status();
}

extern "C" int jz_norm_residual_bwd_workspace_bytes(const jz_norm_residual_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  int64_t groups, per;
  const int rc = norm_shape(d, &groups, &per);
  if (rc == JZ_OK) *bytes = (size_t)slab_count(d->rows, d->channels) * 4 * d->channels * sizeof(float);
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
  const size_t need = (size_t)slab_count(d->rows, d->channels) * 4 * d->channels * sizeof(float);
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
  a.slab = slab_rows(d->rows, d->channels);
  a.slabs = slab_count(d->rows, d->channels);
  a.step = groups == 1 ? std::max(a.slabs, 1) : 1;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (rows) {
    with_types(d, [&](auto te, auto re) {
      with_lanes<false>(d->channels, [&](auto mode, auto th, auto nv) {
        constexpr int M = decltype(mode)::value, TH = decltype(th)::value, NV = decltype(nv)::value;
        auto launch = [&](auto has) { norm_bwd<decltype(te), decltype(re), M, TH, NV, decltype(has)::value><<<(unsigned)a.slabs, TH, 0, st>>>(a); };
        if constexpr (M != TINY && TH < 1024) {  // those that ask ahead
          if (pre && dr_out && branch) return post || gate ? launch(Int<BLOCK>()) : launch(Int<SUM>());
        }
        launch(Int<ANY>());
      });
    });
    if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  }
  if (!a.dw_pre && !a.dw_post && !a.dgate) return JZ_OK;
  const int by_slab = a.slabs > 0 && groups > a.slabs;
  // a wavefront each up to 32 slabs a group: 61 groups of 67 rows, 1001 channels, took the join 6.6 us with a workgroup each, 5.4 so
  const int64_t joins = a.dgate ? by_slab ? a.slabs : groups : 0;
  const int alone = rows && per / a.slab + 2 <= 32;
  const dim3 grid((unsigned)((d->channels + 63) / 64), (unsigned)(2 + (alone ? (joins + JOIN_WAVES - 1) / JOIN_WAVES : joins)));
  with_types(d, [&](auto te, auto) { norm_join<decltype(te)><<<grid, 64 * JOIN_WAVES, 0, st>>>(a, groups, by_slab, alone); });
  return jz::launch_status();
}
