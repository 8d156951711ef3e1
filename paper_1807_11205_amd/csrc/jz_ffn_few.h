// The feed-forward block's forward products for few rows (tokens): C[m][n] = sum over k of A[m][k] B[n][k], both k-contiguous, at most 16 TT rows.
// Included inside jz_ffn.hip's anonymous namespace, behind jz_ffn_gemm.h.
//
// Every weight is read once, so the memory's rate is the bound and what counts is bytes on their way: a wavefront streams 16 rows of weights (16 of each matrix
// where gate and up are made together) straight into the registers that the matrix instruction takes them from, UNROLL steps of 32 k ahead, and the
// wavefronts of a workgroup take k by turns.  Their FP32 sums meet in LDS, in the order of the wavefronts.
// A 16x16x32 matrix instruction with the weights first: lane l supplies row l % 16, k 8 (l / 16) .. + 7, and gets columns (rows of B) 4 (l / 16) .. + 3 of
// token l % 16.
#pragma once

__device__ __forceinline__ f32x4 mfma16(Op8<_Float16> a, Op8<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(Op8<__bf16> a, Op8<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

template <class T, bool GLU, int TT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void ffn_few(GemmArgs a) {
  constexpr int MATS = GLU ? 2 : 1, UNROLL = TT == 1 && WAVES < 16 ? 4 : (TT == 4 ? 2 : 4) / MATS;  // as registers allow
  __shared__ f32x4 sums[WAVES][MATS][TT][64];
  const Product& p = a.p[0];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r16 = lane & 15, k8 = (lane >> 4) * 8;
  const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + r16 < p.N ? n0 + r16 : p.N - 1;  // rows behind the last are computed and not stored
  const T* w[MATS];
#pragma unroll
  for (int i = 0; i < MATS; ++i) w[i] = static_cast<const T*>(p.b[i]) + n * p.ldb;
  const T* x[TT];
#pragma unroll
  for (int j = 0; j < TT; ++j) x[j] = static_cast<const T*>(p.a[0]) + (j * 16 + r16 < p.M ? j * 16 + r16 : 0) * p.lda;
  f32x4 acc[MATS][TT];
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Weights are asked for a turn ahead; the rows of A, which all workgroups share and the caches hold, in their own turn.
  constexpr int64_t DEPTH = UNROLL * 32, TURN = DEPTH * WAVES;
  const int64_t whole = p.K / DEPTH * DEPTH;
  Op8<T> cur[UNROLL][MATS], next[UNROLL][MATS];
  auto weights = [&](Op8<T>(&to)[UNROLL][MATS], int64_t k0) {  // whole steps only
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < MATS; ++i) to[u][i] = load8(w[i] + k0 + u * 32 + k8);
  };
  auto turn = [&](Op8<T>(&have)[UNROLL][MATS], Op8<T>(&ask)[UNROLL][MATS], int64_t k0) {
    Op8<T> xs[UNROLL][TT];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int j = 0; j < TT; ++j) xs[u][j] = load8(x[j] + k0 + u * 32 + k8);
    if (k0 + TURN < whole) weights(ask, k0 + TURN);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u)
#pragma unroll
      for (int i = 0; i < MATS; ++i)
#pragma unroll
        for (int j = 0; j < TT; ++j) acc[i][j] = mfma16(have[u][i], xs[u][j], acc[i][j]);
  };
  int64_t k0 = wave * DEPTH;
  if (k0 < whole) weights(cur, k0);
  while (k0 < whole) {
    turn(cur, next, k0);
    k0 += TURN;
    if (k0 >= whole) break;
    turn(next, cur, k0);
    k0 += TURN;
  }
  // what is left, 32 k at a time, one wavefront each
  for (int64_t k = whole + wave * 32; k < p.K; k += WAVES * 32) {
    const int64_t left = p.K - k - k8;
    const int m = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    Op8<T> ww[MATS], xx[TT];
#pragma unroll
    for (int i = 0; i < MATS; ++i) {
      ww[i] = {};
      if (m > 0) ww[i] = load8(w[i] + k + k8, m);
    }
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      xx[j] = {};
      if (m > 0) xx[j] = load8(x[j] + k + k8, m);
    }
#pragma unroll
    for (int i = 0; i < MATS; ++i)
#pragma unroll
      for (int j = 0; j < TT; ++j) acc[i][j] = mfma16(ww[i], xx[j], acc[i][j]);
  }
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) sums[wave][i][j][lane] = acc[i][j];
  __syncthreads();
  for (int s = t; s < TT * 64; s += 64 * WAVES) {  // one lane a token and four columns
    const int j = s >> 6, l = s & 63;
    f32x4 v[MATS];
#pragma unroll
    for (int i = 0; i < MATS; ++i) {
      v[i] = sums[0][i][j][l];
#pragma unroll
      for (int q = 1; q < WAVES; ++q) v[i] += sums[q][i][j][l];
    }
    const int64_t m = j * 16 + (l & 15);
    if (m >= p.M) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t col = n0 + (l >> 4) * 4 + e;
      if (col >= p.N) break;
      if constexpr (GLU) {
        static_cast<T*>(p.c)[m * p.ldc + col] = (T)(act_fwd(a.act, v[0][e]) * v[MATS - 1][e]);
        if (a.out0) {
          static_cast<T*>(a.out0)[m * p.N + col] = (T)v[0][e];
          static_cast<T*>(a.out1)[m * p.N + col] = (T)v[MATS - 1][e];
        }
      } else {
        static_cast<T*>(p.c)[m * p.ldc + col] = (T)v[0][e];
      }
    }
  }
}
