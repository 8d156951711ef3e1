// Global norm of the gradients of many tensors, and clipping by it (include/jz.h: jz_grad_norm, jz_grad_clip).
//
//   norm = sqrt(sum over tensors and elements of g^2) / S,   out = RNE(c g),  c = max_norm / norm where norm > max_norm, else 1
//
// Two launches over a table of chunks.  The first leaves one partial sum of squares a workgroup; the second adds those up in every
// workgroup (in one order, so all of them have the same bits), forms c and scales.  What bounds it: memory.  A gradient is read
// twice and written once, and the second pass takes the chunks in the reverse order, so that it begins with what the first
// read last and the 256 MiB last-level cache still holds.  25.6 M FP16 elements 33 us, 600 M of BF16 728 us (4.9 TB/s of the three passes), 400 000 7 to 9 us (launches).
//
// Numbers: eight squares are added in FP32, which holds the square of an FP16 value exactly; everything above that is FP64.  BF16 and FP32
// values whose squares leave the FP32 range are squared again in FP64, so the sum is not finite exactly if a gradient is not.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "jz_internal.h"

namespace {

#include "jz_vec.h"

constexpr uint64_t CLIP_MAGIC = 0x70696c6367726164ull;
constexpr int CLIP_THREADS = 256;
constexpr int CLIP_GRID = 2048;        // workgroups at most: 8 a compute unit

struct ClipChunk {
  const void* in;
  void* out;
  int count, dtype;
};

// Elements of a chunk: eight vectors of eight a lane, or one where a list is so short that its chunks would not fill the chip (FP16, 24 tensors, calls on the same gradients
// one behind the other: 400 000 elements 8.4 us with the longer, 7.2 with the shorter; 1 million 9.3 and 7.4, 1.5 million 8.8 and 8.4; waited for after every call 21.3 and 19.4, 21.9 and
// 19.9, 21.3 and 20.8.  2 million: 9.2 with either, 4.1 million 10.9 and 12.3).
int64_t chunk_of(int64_t elements) { return elements <= int64_t(3) << 19 ? 2048 : 16384; }

struct ClipLayout {
  int64_t chunk = 0, n_chunks = 0;
  size_t off_chunks = 0, static_bytes = 0, off_psum = 0, total = 0;
  int grid = 0;
};

inline size_t up256(size_t n) { return (n + 255) & ~size_t(255); }
inline int elem_bytes(int dtype) { return dtype == JZ_F32 ? 4 : 2; }

int clip_layout(const jz_grad_list* gl, ClipLayout* L) {
  if (!gl) return JZ_ERR_NULL;
  if (gl->num_tensors < 0) return JZ_ERR_SHAPE;
  if (gl->num_tensors > 0 && (!gl->grads || !gl->numel || !gl->dtypes)) return JZ_ERR_NULL;
  if (gl->num_tensors >= (int64_t(1) << 24)) return JZ_ERR_UNSUPPORTED;
  int64_t elements = 0, chunks = 0;
  for (int64_t t = 0; t < gl->num_tensors; ++t) {
    const int64_t n = gl->numel[t];
    if (n < 0 || gl->dtypes[t] < JZ_F16 || gl->dtypes[t] > JZ_F32) return JZ_ERR_SHAPE;
    if (n >= (int64_t(1) << 44)) return JZ_ERR_UNSUPPORTED;
    if (n == 0) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(gl->grads[t]), o = gl->out ? reinterpret_cast<uintptr_t>(gl->out[t]) : a;
    if (!a || !o) return JZ_ERR_NULL;
    if (((a | o) & (elem_bytes(gl->dtypes[t]) - 1)) != 0) return JZ_ERR_ALIGN;
    elements += n;
    if (elements >= (int64_t(1) << 44)) return JZ_ERR_UNSUPPORTED;
  }
  L->chunk = chunk_of(elements);
  for (int64_t t = 0; t < gl->num_tensors; ++t) chunks += (gl->numel[t] + L->chunk - 1) / L->chunk;
  if (chunks >= (int64_t(1) << 30)) return JZ_ERR_UNSUPPORTED;
  L->n_chunks = chunks;
  L->grid = (int)std::min<int64_t>(chunks, CLIP_GRID);
  size_t o = up256(64);
  L->off_chunks = o;
  o = up256(o + sizeof(ClipChunk) * (size_t)chunks);
  L->static_bytes = o;
  L->off_psum = o;
  L->total = up256(o + sizeof(double) * CLIP_GRID);
  return JZ_OK;
}

uint64_t list_checksum(const jz_grad_list* gl) {
  uint64_t h = 1469598103934665603ull;
  auto mix = [&](uint64_t v) {
    h = (h ^ v) * 0x9e3779b97f4a7c15ull;
    h ^= h >> 32;
  };
  mix((uint64_t)gl->num_tensors);
  for (int64_t t = 0; t < gl->num_tensors; ++t) {
    mix(reinterpret_cast<uintptr_t>(gl->grads[t]));
    mix(reinterpret_cast<uintptr_t>(gl->out ? gl->out[t] : gl->grads[t]));
    mix((uint64_t)gl->numel[t]);
    mix((uint64_t)gl->dtypes[t]);
  }
  return h;
}

// ---- device -------------------------------------------------------------------------------------------------------------
struct ClipArgs {
  const uint64_t* header;
  const ClipChunk* chunks;
  double* psum;
  uint64_t checksum;
  int n_chunks, grid;
  float loss_scale;
  const jz_loss_scale_state* state;
  float max_norm;
  float* norm;
  int* found_inf;
};
__device__ __forceinline__ bool list_ok(const ClipArgs& a) { return a.header[0] == CLIP_MAGIC && a.header[1] == a.checksum; }

// the sum of eight squares
template <class T>
__device__ __forceinline__ double sumsq8(f32x8 v) {
  const f32x8 q = v * v;
  const float s = ((q[0] + q[1]) + (q[2] + q[3])) + ((q[4] + q[5]) + (q[6] + q[7]));
  if constexpr (sizeof(T) == 2 && !__is_same(T, __bf16)) return s;  // FP16: from 2^-48 to 2^35
  else {
    // squares from 2^-100 on lose nothing that FP32 keeps; smaller sums, and those that overflowed, again in FP64
    if (s >= 0x1p-100f && s < INFINITY) return s;
    double d = 0.;
#pragma unroll
    for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
    return d;
  }
}

template <class T>
__device__ __forceinline__ double chunk_sumsq(const T* __restrict__ p, int n, int lane) {
  double s = 0.;
  int i = lane * 8;
  // four loads in flight
  for (; i + 3 * CLIP_THREADS * 8 + 8 <= n; i += 4 * CLIP_THREADS * 8) {
    typename Vec8<T>::V v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = load8(p + i + k * CLIP_THREADS * 8);
#pragma unroll
    for (int k = 0; k < 4; ++k) s += sumsq8<T>(widen8<T>(v[k]));
  }
  for (; i < n; i += CLIP_THREADS * 8) s += sumsq8<T>(widen8<T>(load8(p + i, n - i)));
  return s;
}

// c g in FP32, from a factor in FP32 or, where that would be below FP32's smallest normal number (exploded gradients of FP32 or BF16), in FP64
__device__ __forceinline__ f32x8 scaled8(f32x8 v, float c) { return v * c; }
__device__ __forceinline__ f32x8 scaled8(f32x8 v, double c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)((double)v[i] * c);
  return v;
}
template <class T, class F>
__device__ __forceinline__ void chunk_scale(const T* in, T* out, int n, F c, int lane) {
  int i = lane * 8;
  for (; i + 3 * CLIP_THREADS * 8 + 8 <= n; i += 4 * CLIP_THREADS * 8) {
    typename Vec8<T>::V v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = load8(in + i + k * CLIP_THREADS * 8);
#pragma unroll
    for (int k = 0; k < 4; ++k) store8(out + i + k * CLIP_THREADS * 8, narrow8<T>(scaled8(widen8<T>(v[k]), c)));
  }
  for (; i < n; i += CLIP_THREADS * 8) store8(out + i, narrow8<T>(scaled8(widen8<T>(load8(in + i, n - i)), c)), n - i);
}
template <class T>
__device__ __forceinline__ void chunk_copy(const T* in, T* out, int n, int lane) {  // bit for bit: a NaN keeps its payload
  for (int i = lane * 8; i < n; i += CLIP_THREADS * 8) store8(out + i, load8(in + i, n - i), n - i);
}

// the sum over a workgroup, in one order, in every lane
__device__ __forceinline__ double block_sum(double s, double* lds) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(CLIP_THREADS) void grad_sumsq(ClipArgs a) {
  __shared__ double lds[CLIP_THREADS / 64];
  if (!list_ok(a)) return;
  double s = 0.;
  for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
    const ClipChunk r = a.chunks[c];
    if (r.dtype == JZ_F16) s += chunk_sumsq(static_cast<const _Float16*>(r.in), r.count, threadIdx.x);
    else if (r.dtype == JZ_BF16) s += chunk_sumsq(static_cast<const __bf16*>(r.in), r.count, threadIdx.x);
    else s += chunk_sumsq(static_cast<const float*>(r.in), r.count, threadIdx.x);
  }
  s = block_sum(s, lds);
  if (threadIdx.x == 0) a.psum[blockIdx.x] = s;
}

// The norm from the partial sums, the same bits in every workgroup; workgroup 0 writes it and the flag.  Returns the factor.
__device__ __forceinline__ double join_norm(const ClipArgs& a, double* lds) {
  double s = 0.;
#pragma unroll
  for (int k = 0; k < CLIP_GRID / CLIP_THREADS; ++k) {
    const int i = k * CLIP_THREADS + threadIdx.x;
    if (i < a.grid) s += a.psum[i];
  }
  s = block_sum(s, lds);
  const double scale = a.state ? (double)a.state->scale : (double)a.loss_scale;
  const double norm = sqrt(s) / scale;
  const bool bad = !(s < INFINITY);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.norm = (float)norm;
    *a.found_inf = bad ? 1 : 0;
  }
  return !bad && norm > (double)a.max_norm ? (double)a.max_norm / norm : 1.;
}

__global__ __launch_bounds__(CLIP_THREADS) void grad_norm_final(ClipArgs a) {
  __shared__ double lds[CLIP_THREADS / 64];
  if (!list_ok(a)) {
    if (threadIdx.x == 0) {
      *a.norm = NAN;
      *a.found_inf = -1;
    }
    return;
  }
  join_norm(a, lds);
}

// 64 registers a lane, so that all of the workgroups are on the chip at once (the FP64 form would take 70)
__global__ __launch_bounds__(CLIP_THREADS, 8) void grad_scale(ClipArgs a) {
  __shared__ double lds[CLIP_THREADS / 64];
  if (!list_ok(a)) {
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      *a.norm = NAN;
      *a.found_inf = -1;
    }
    return;
  }
  const double exact = join_norm(a, lds);
  const float f = (float)exact;
  const bool tiny = exact < 0x1p-126 && exact > 0.;
  for (int c = a.n_chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
    const ClipChunk r = a.chunks[c];
    if (f == 1.f && r.in == r.out) continue;
    if (r.dtype == JZ_F32) {
      if (f == 1.f) chunk_copy(static_cast<const float*>(r.in), static_cast<float*>(r.out), r.count, threadIdx.x);
      else if (tiny) chunk_scale(static_cast<const float*>(r.in), static_cast<float*>(r.out), r.count, exact, threadIdx.x);
      else chunk_scale(static_cast<const float*>(r.in), static_cast<float*>(r.out), r.count, f, threadIdx.x);
    } else if (f == 1.f) {
      chunk_copy(static_cast<const _Float16*>(r.in), static_cast<_Float16*>(r.out), r.count, threadIdx.x);
    } else if (r.dtype == JZ_F16) {
      chunk_scale(static_cast<const _Float16*>(r.in), static_cast<_Float16*>(r.out), r.count, f, threadIdx.x);  // of a tiny factor zeros, in FP16 as in FP32
    } else if (tiny) {
      chunk_scale(static_cast<const __bf16*>(r.in), static_cast<__bf16*>(r.out), r.count, exact, threadIdx.x);
    } else {
      chunk_scale(static_cast<const __bf16*>(r.in), static_cast<__bf16*>(r.out), r.count, f, threadIdx.x);
    }
  }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
// An output is its own gradient or touches nothing that is read or written.
int list_aliases(const jz_grad_list* gl, const void* ws, size_t ws_bytes) {
  struct Span {
    uintptr_t lo, hi;
    int64_t tensor;
    bool out;
  };
  std::vector<Span> spans;
  for (int64_t t = 0; t < gl->num_tensors; ++t) {
    if (gl->numel[t] == 0) continue;
    const uintptr_t n = (uintptr_t)gl->numel[t] * elem_bytes(gl->dtypes[t]);
    const uintptr_t a = reinterpret_cast<uintptr_t>(gl->grads[t]), o = gl->out ? reinterpret_cast<uintptr_t>(gl->out[t]) : a;
    spans.push_back({o, o + n, t, true});
    if (o != a) spans.push_back({a, a + n, t, false});
    if (jz::overlaps(ws, ws_bytes, gl->grads[t], n) || jz::overlaps(ws, ws_bytes, reinterpret_cast<const void*>(o), n)) return JZ_ERR_ALIAS;
  }
  std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.lo < y.lo; });
  uintptr_t end_out = 0, end_any = 0;  // how far outputs, and anything, reach so far
  for (const Span& s : spans) {
    if (s.lo < end_out || (s.out && s.lo < end_any)) return JZ_ERR_ALIAS;
    end_any = std::max(end_any, s.hi);
    if (s.out) end_out = std::max(end_out, s.hi);
  }
  return JZ_OK;
}

int clip_check(const jz_grad_list* gl, float loss_scale, const jz_loss_scale_state* state, const float* norm, const int* found_inf,
               void* ws, size_t ws_bytes, ClipLayout* L) {
  const int rc = clip_layout(gl, L);
  if (rc != JZ_OK) return rc;
  if (!norm || !found_inf) return JZ_ERR_NULL;
  if (!state && !(loss_scale > 0.f && loss_scale < INFINITY)) return JZ_ERR_SHAPE;
  if (!ws || ws_bytes < L->total) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(ws) || (reinterpret_cast<uintptr_t>(norm) & 3) || (reinterpret_cast<uintptr_t>(found_inf) & 3) || (reinterpret_cast<uintptr_t>(state) & 7))
    return JZ_ERR_ALIGN;
  if (jz::overlaps(norm, 4, ws, ws_bytes) || jz::overlaps(found_inf, 4, ws, ws_bytes) || jz::overlaps(norm, 4, found_inf, 4) ||
      jz::overlaps(state, 8, ws, ws_bytes) || jz::overlaps(state, 8, norm, 4) || jz::overlaps(state, 8, found_inf, 4))
    return JZ_ERR_ALIAS;
  return JZ_OK;
}

ClipArgs clip_args(const jz_grad_list* gl, const ClipLayout& L, float max_norm, float loss_scale, const jz_loss_scale_state* state, float* norm,
                   int* found_inf, void* ws) {
  char* b = static_cast<char*>(ws);
  return ClipArgs{reinterpret_cast<const uint64_t*>(b), reinterpret_cast<const ClipChunk*>(b + L.off_chunks), reinterpret_cast<double*>(b + L.off_psum),
                  list_checksum(gl), (int)L.n_chunks, L.grid, loss_scale, state, max_norm, norm, found_inf};
}

int prepare(const jz_grad_list* gl, const ClipLayout& L, void* ws, size_t ws_bytes, hipStream_t st) {
  const int rc = list_aliases(gl, ws, ws_bytes);
  if (rc != JZ_OK) return rc;
  std::vector<char> host(L.static_bytes, 0);
  uint64_t* hdr = reinterpret_cast<uint64_t*>(host.data());
  hdr[0] = CLIP_MAGIC;
  hdr[1] = list_checksum(gl);
  ClipChunk* c = reinterpret_cast<ClipChunk*>(host.data() + L.off_chunks);
  for (int64_t t = 0; t < gl->num_tensors; ++t) {
    const int b = elem_bytes(gl->dtypes[t]);
    const char* in = static_cast<const char*>(gl->grads[t]);
    char* out = gl->out ? static_cast<char*>(gl->out[t]) : const_cast<char*>(in);
    for (int64_t at = 0; at < gl->numel[t]; at += L.chunk)
      *c++ = ClipChunk{in + at * b, out + at * b, (int)std::min(L.chunk, gl->numel[t] - at), gl->dtypes[t]};
  }
  if (hipMemcpyAsync(ws, host.data(), L.static_bytes, hipMemcpyHostToDevice, st) != hipSuccess) return JZ_ERR_LAUNCH;
  return hipStreamSynchronize(st) == hipSuccess ? JZ_OK : JZ_ERR_LAUNCH;
}

}  // namespace

extern "C" int jz_grad_clip_workspace_bytes(const jz_grad_list* gl, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  ClipLayout L;
  const int rc = clip_layout(gl, &L);
  if (rc == JZ_OK) *bytes = L.total;
  return rc;
}

extern "C" int jz_grad_clip_prepare(const jz_grad_list* gl, void* ws, size_t ws_bytes, void* hip_stream) {
  ClipLayout L;
  const int rc = clip_layout(gl, &L);
  if (rc != JZ_OK) return rc;
  if (!ws || ws_bytes < L.total) return JZ_ERR_WORKSPACE;
  if (!jz::aligned16(ws)) return JZ_ERR_ALIGN;
  try {
    return prepare(gl, L, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
  } catch (const std::bad_alloc&) {  // host memory for the table
    return JZ_ERR_LAUNCH;
  }
}

extern "C" int jz_grad_norm(const jz_grad_list* gl, float loss_scale, const jz_loss_scale_state* state_dev, float* norm_dev, int* found_inf_dev,
                            void* ws, size_t ws_bytes, void* hip_stream) {
  ClipLayout L;
  const int rc = clip_check(gl, loss_scale, state_dev, norm_dev, found_inf_dev, ws, ws_bytes, &L);
  if (rc != JZ_OK) return rc;
  const ClipArgs a = clip_args(gl, L, INFINITY, loss_scale, state_dev, norm_dev, found_inf_dev, ws);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (L.grid > 0) {
    grad_sumsq<<<L.grid, CLIP_THREADS, 0, st>>>(a);
    if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  }
  grad_norm_final<<<1, CLIP_THREADS, 0, st>>>(a);
  return jz::launch_status();
}

extern "C" int jz_grad_clip(const jz_grad_list* gl, float max_norm, float loss_scale, const jz_loss_scale_state* state_dev, float* norm_dev,
                            int* found_inf_dev, void* ws, size_t ws_bytes, void* hip_stream) {
  ClipLayout L;
  const int rc = clip_check(gl, loss_scale, state_dev, norm_dev, found_inf_dev, ws, ws_bytes, &L);
  if (rc != JZ_OK) return rc;
  if (!(max_norm >= 0.f)) return JZ_ERR_SHAPE;
  const ClipArgs a = clip_args(gl, L, max_norm, loss_scale, state_dev, norm_dev, found_inf_dev, ws);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (L.grid > 0) {
    grad_sumsq<<<L.grid, CLIP_THREADS, 0, st>>>(a);
    if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  }
  grad_scale<<<L.grid > 0 ? L.grid : 1, CLIP_THREADS, 0, st>>>(a);
  return jz::launch_status();
}
