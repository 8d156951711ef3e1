// Eight elements of FP16, BF16 or FP32 to and from FP32 registers, for kernels that stream rows or flat buffers of any length: the
// accesses are typed as aligned to one element, so a row of odd length is still moved 16 bytes at a time (global memory takes
// unaligned vector accesses; they cost a second line where they cross one).  Included inside a kernel file's anonymous namespace.
#pragma once

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T>
struct Vec8;
template <>
struct Vec8<_Float16> {
  typedef _Float16 V __attribute__((ext_vector_type(8)));
  typedef V U __attribute__((aligned(2)));
};
template <>
struct Vec8<__bf16> {
  typedef __bf16 V __attribute__((ext_vector_type(8)));
  typedef V U __attribute__((aligned(2)));
};
template <>
struct Vec8<float> {
  typedef f32x8 V;
  typedef V U __attribute__((aligned(4)));
};

template <class T>
__device__ __forceinline__ typename Vec8<T>::V load8(const T* p) {
  return *reinterpret_cast<const typename Vec8<T>::U*>(p);
}
template <class T>
__device__ __forceinline__ void store8(T* p, typename Vec8<T>::V v) {
  *reinterpret_cast<typename Vec8<T>::U*>(p) = v;
}
// past the caches: for results of half of the last-level cache and more, of which they would keep little
constexpr size_t STREAM_BYTES = size_t(128) << 20;
template <class T>
__device__ __forceinline__ void stream8(T* p, typename Vec8<T>::V v) {
  __builtin_nontemporal_store(v, reinterpret_cast<typename Vec8<T>::U*>(p));
}
template <class T>
__device__ __forceinline__ f32x8 widen8(typename Vec8<T>::V v) {
  return __builtin_convertvector(v, f32x8);
}
template <class T>
__device__ __forceinline__ typename Vec8<T>::V narrow8(f32x8 v) {  // one rounding to nearest even
  return __builtin_convertvector(v, typename Vec8<T>::V);
}
// the first n of eight elements, zeros behind them
template <class T>
__device__ __forceinline__ typename Vec8<T>::V load8(const T* p, int n) {
  if (n >= 8) return load8(p);
  typename Vec8<T>::V v = {};
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) v[i] = p[i];
  return v;
}
template <class T>
__device__ __forceinline__ void store8(T* p, typename Vec8<T>::V v, int n) {
  if (n >= 8) {
    store8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 7; ++i)
    if (i < n) p[i] = v[i];
}
