// How the matrix-product kernels with LDS-direct loads order a tile's work.  Included inside a kernel file's anonymous namespace, behind jz_lds_dma.h.
#pragma once

#define JZ_LDS __attribute__((address_space(3)))

// Everything has landed that this wavefront asked for, and every wavefront is past its reads: both sides are ordinary accesses, which the
// fences keep in place.
__device__ __forceinline__ void all_landed() {
  __builtin_amdgcn_sched_barrier(0);
  wait_vmcnt<0>();
  lds_wait<0>();
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  __builtin_amdgcn_sched_barrier(0);
}

// The same without a wait for what is on its way from memory.
__device__ __forceinline__ void lds_meet() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The order of a step's instructions: between one matrix instruction and the next a read of LDS or a load.  (In the compiler's order, all reads first, 8192 rows, 2048 ->
// 5632 features take 10 % longer.)
template <int MULTIPLY, int READ, int LOAD>
__device__ __forceinline__ void spread_out() {
  constexpr int OTHER = READ + LOAD;
  static_for<0, MULTIPLY>([&](auto I) {
    constexpr int i = decltype(I)::value, from = i * OTHER / MULTIPLY, to = (i + 1) * OTHER / MULTIPLY;
    constexpr int reads = (to < READ ? to : READ) - (from < READ ? from : READ), loads = to - from - reads;
    if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
    if constexpr (loads > 0) __builtin_amdgcn_sched_group_barrier(0x10, loads, 0);
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
  });
}
