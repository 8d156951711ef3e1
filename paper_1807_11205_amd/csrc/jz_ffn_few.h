// The feed-forward block's forward products for few rows (tokens): C[m][n] = sum over k of A[m][k] B[n][k], both k-contiguous, at most 16 TT rows.
// Included inside jz_ffn.hip's anonymous namespace, behind jz_ffn_gemm.h.
//
// Every weight is read once, so with many columns the memory's rate is the bound, and with fewer what a compute unit can bring in: 16 columns (of each matrix,
// where gate and up are made together) are a workgroup's, whose wavefronts take k by turns, and their FP32 sums meet in LDS in the order of the wavefronts.
// A 16x16x32 matrix instruction with the weights first: lane l supplies row l % 16, k 8 (l / 16) .. + 7, and gets columns (rows of B) 4 (l / 16) .. + 3 of
// token l % 16.
#pragma once

__device__ __forceinline__ f32x4 mfma16(Op8<_Float16> a, Op8<_Float16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(Op8<__bf16> a, Op8<__bf16> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// The wavefronts' sums [wave][matrix][16 tokens][lane] added in their order, and the results.
template <class T, bool GLU, int TT, int WAVES>
__device__ __forceinline__ void few_finish(const GemmArgs& a, const Product& p, int64_t n0, const JZ_LDS f32x4* sums, int t) {
  constexpr int MATS = GLU ? 2 : 1;
  for (int s = t; s < TT * 64; s += 64 * WAVES) {  // one lane a token and four columns
    const int j = s >> 6, l = s & 63;
    f32x4 v[MATS];
#pragma unroll
    for (int i = 0; i < MATS; ++i) {
      v[i] = sums[(i * TT + j) * 64 + l];
#pragma unroll 4
      for (int q = 1; q < WAVES; ++q) v[i] += sums[((q * MATS + i) * TT + j) * 64 + l];
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

// Any sizes, any alignment: weights go straight into the registers that the matrix instruction takes them from, UNROLL steps of 32 k ahead.  Slower than the next kernel at
// aligned sizes (BF16, 24 rows, 5632 -> 2048 features 17.0 us and 7.2), and slower still where rows are not: both products of 24 rows, 2048 -> 5632 -> 2048 features, take 20 us
// there, 38 at 2046 -> 5630 -> 2046 (rows on 4 bytes) and 105 at 2047 -> 5631 -> 2047 (on 2).
template <class T, bool GLU, int TT, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void ffn_few_any(GemmArgs a) {
  constexpr int MATS = GLU ? 2 : 1, UNROLL = TT == 1 && WAVES < 16 ? 4 : (TT == 4 ? 2 : 4) / MATS;  // as registers allow
  __shared__ f32x4 sums[WAVES * MATS * TT * 64];
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
    weights(ask, k0 + TURN < whole ? k0 + TURN : k0);  // without a branch, in which the compiler would lose count of the loads on their way
    __builtin_amdgcn_sched_barrier(0);                 // all are asked for before the first is waited for
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
    for (int j = 0; j < TT; ++j) sums[((wave * MATS + i) * TT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  few_finish<T, GLU, TT, WAVES>(a, p, n0, (const JZ_LDS f32x4*)sums, t);
}

// Rows that are multiples of 8: LDS-direct loads of 8 rows x 128 bytes, whole lines, into places of the wavefront's own, so that it waits for nobody.  (Loads in
// the matrix instruction's layout, 16 rows x 64 bytes, bring a compute unit 17 bytes a clock.)  FP16, one row, 4096 -> 12288 -> 4096 forward in both products:
// 53 us, the weights at 5.7 TB/s (other weights every time: 56 us); BF16, 2048 -> 5632 -> 2048 features: 21 us for 24 rows, 26 for 40, 32 for 64.  A stage is 64 CH k of the weights' and the tokens' rows, chunk c of a row at c ^ (row / 2 % 8); two stages.
template <class T, bool GLU, int TT, int WAVES, int CH>
__global__ __launch_bounds__(64 * WAVES) void ffn_few(GemmArgs a) {
  constexpr int MATS = GLU ? 2 : 1, ROWS = 16 * (MATS + TT), CHUNK = ROWS * 128, STAGE = CHUNK * CH;
  __shared__ __attribute__((aligned(1024))) unsigned char s0[WAVES * STAGE], s1[WAVES * STAGE];
  const Product& p = a.p[0];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  // the first and the second 8 of 16 rows: which elements of 64 an LDS-direct load brings to position lane % 8 of row lane / 8
  const int row = lane >> 3;
  const unsigned k8[2] = {((lane & 7u) ^ (row >> 1)) * 8u, ((lane & 7u) ^ (4 + (row >> 1))) * 8u};
  const unsigned off_w = (unsigned)(row * p.ldb) * 2, off_x = (unsigned)(row * p.lda) * 2;
  const int stages = (int)((p.K + 64 * CH - 1) / (64 * CH));
  auto fetch = [&](unsigned char* s, int j) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t k0 = ((int64_t)j * CH + c) * 64;
      const bool wanted = k0 < p.K;
      auto at = [&](int h, int64_t ld, unsigned off) { return (off + (unsigned)(h * 8 * ld * 2) + k8[h & 1] * 2) | (k8[h & 1] >= p.K - k0 ? 0x80000000u : 0u); };
      auto span = [&](int64_t rows, int64_t ld) {  // bytes from the place on; nothing behind the end
        const int64_t n = ((rows - 1) * ld + p.K - k0) * 2;
        return wanted ? (int)(n < 0x7ffffff0 ? n : 0x7ffffff0) : 0;
      };
      unsigned char* to = s + wave * STAGE + c * CHUNK;
#pragma unroll
      for (int i = 0; i < MATS; ++i) {
        const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(static_cast<const T*>(p.b[i]) + n0 * p.ldb + (wanted ? k0 : 0)), 0, span(p.N - n0, p.ldb), 0x00020000);
#pragma unroll
        for (int h = 0; h < 2; ++h) jz_dma16(r, (lds_byte*)to + (i * 2 + h) * 1024, at(h, p.ldb, off_w));
      }
      const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(static_cast<const T*>(p.a[0]) + (wanted ? k0 : 0)), 0, span(p.M, p.lda), 0x00020000);
#pragma unroll
      for (int h = 0; h < 2 * TT; ++h) jz_dma16(r, (lds_byte*)to + (MATS * 2 + h) * 1024, at(h, p.lda, off_x));
    }
  };
  f32x4 acc[MATS][TT];
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto turn = [&](unsigned char* s, int j) {
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<CH * 2 * (MATS + TT)>();  // this stage has landed; the other one's loads were asked for later
    __builtin_amdgcn_sched_barrier(0);
    const JZ_LDS unsigned char* from = (const JZ_LDS unsigned char*)s + wave * STAGE + r16 * 128;
    Op8<T> w[CH][2][MATS], x[CH][2][TT];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = c * CHUNK + (((u * 4 + (lane >> 4)) ^ ((lane >> 1) & 7)) * 16);
#pragma unroll
        for (int i = 0; i < MATS; ++i) w[c][u][i] = *reinterpret_cast<const JZ_LDS Op8<T>*>(from + at + i * 2048);
#pragma unroll
        for (int k = 0; k < TT; ++k) x[c][u][k] = *reinterpret_cast<const JZ_LDS Op8<T>*>(from + at + (MATS + k) * 2048);
      }
    __builtin_amdgcn_sched_barrier(0);
    lds_wait<0>();  // read, before the stage is filled again
    __builtin_amdgcn_sched_barrier(0);
    fetch(s, j + 2 * WAVES);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < MATS; ++i)
#pragma unroll
          for (int k = 0; k < TT; ++k) acc[i][k] = mfma16(w[c][u][i], x[c][u][k], acc[i][k]);
  };
  fetch(s0, wave);
  fetch(s1, wave + WAVES);
  for (int j = wave; j < stages; j += 2 * WAVES) {
    turn(s0, j);
    turn(s1, j + WAVES);  // behind the end: zeros
  }
  wait_vmcnt<0>();
  __syncthreads();  // nothing is on its way into LDS any more
  static_assert(MATS * TT * 1024 <= STAGE, "the sums take a stage's place");
  JZ_LDS f32x4* const sums = (JZ_LDS f32x4*)s0;
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) sums[((wave * MATS + i) * TT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  few_finish<T, GLU, TT, WAVES>(a, p, n0, sums, t);
}
