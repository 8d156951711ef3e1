// Products of codes for few rows (tokens), at most 16 TT of them.  Included inside jz_i8.hip's anonymous namespace, behind jz_ffn_gemm.h and jz_mm_tile.h.
//
// Every weight is read once, and the memory's rate is the bound.  16 channels (of each matrix, where gate and up are made together) are a workgroup's, whose wavefronts take k by
// turns with places in LDS of their own, filled by LDS-direct loads of 8 rows x 128 bytes; a place is CH such pieces of the 16 rows, chunk c of a row at c ^ (row / 2 % 8), and
// there are two.  The sums, whole numbers, meet in LDS.  A 16x16x64 matrix instruction with the weights first: lane l supplies row l % 16, k 16 (l / 16) .. + 15, and gets channels
// 4 (l / 16) .. + 3 of token l % 16.
// QUANTIZE: up to four short rows get their codes in every workgroup, while the first weights are on their way, instead of in a launch of their own.
// FP16, one row, 4096 -> 12288: 14.5 us (50 MB; 24 with a launch for the codes and 64 x 64 tiles), of which about five pass before the first weights arrive.  BF16, 24 rows, 2048 -> 5632 -> 2048:
// four launches of 4 to 9 us.  (Places of four pieces: 19.8 us for the first; 19.3 instead of 21.3 for 8192 -> 8192.)
#pragma once

struct FewArgs {
  const signed char *q, *w[2];  // codes of the tokens (not QUANTIZE) and of the weights
  const float *sx, *sw[2];
  const void* x;                // QUANTIZE: the rows themselves
  void* y;
  int64_t M, N, K, pitch, ldx, ldy;
  int act;
};
constexpr int FEW_CODES = 8192;  // bytes of codes that a workgroup makes itself

template <class X, class Y, bool GLU, int TT, int WAVES, int CH, bool QUANTIZE>
__global__ __launch_bounds__(64 * WAVES) void i8_few(FewArgs a) {
  constexpr int MATS = GLU ? 2 : 1, FROM_X = QUANTIZE ? 0 : TT, ROWS = 16 * (MATS + FROM_X), PIECE = ROWS * 128, PLACE = PIECE * CH, THREADS = 64 * WAVES;
  __shared__ __attribute__((aligned(1024))) unsigned char s0[WAVES * PLACE], s1[WAVES * PLACE];
  __shared__ __attribute__((aligned(16))) unsigned char codes[QUANTIZE ? FEW_CODES : 16];
  __shared__ unsigned most[4];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), r16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int row = lane >> 3;
  const unsigned k16[2] = {((lane & 7u) ^ (row >> 1)) * 16u, ((lane & 7u) ^ (4 + (row >> 1))) * 16u};  // of the first and the second 8 of 16 rows
  const unsigned off = (unsigned)(row * a.pitch);
  const int pieces = (int)((a.pitch + 127) / 128), places = (pieces + CH - 1) / CH;
  auto fetch = [&](unsigned char* s, int j) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int64_t k0 = ((int64_t)j * CH + c) * 128;
      const bool wanted = k0 < a.pitch;
      auto at = [&](int h) { return (off + (unsigned)(h * 8 * a.pitch) + k16[h & 1]) | ((int64_t)k16[h & 1] >= a.pitch - k0 ? 0x80000000u : 0u); };
      auto span = [&](int64_t rows) { return wanted ? (int)((rows < 65536 / 8 ? rows : 65536 / 8) * a.pitch - k0) : 0; };  // more rows than a workgroup reads, less than 2^31 bytes
      unsigned char* to = s + wave * PLACE + c * PIECE;
#pragma unroll
      for (int i = 0; i < MATS; ++i) {
        const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(a.w[i] + n0 * a.pitch + (wanted ? k0 : 0)), 0, span(a.N - n0), 0x00020000);
#pragma unroll
        for (int h = 0; h < 2; ++h) jz_dma16(r, (lds_byte*)to + (i * 2 + h) * 1024, at(h));
      }
      if constexpr (!QUANTIZE) {
        const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(a.q + (wanted ? k0 : 0)), 0, span(a.M), 0x00020000);
#pragma unroll
        for (int h = 0; h < 2 * TT; ++h) jz_dma16(r, (lds_byte*)to + (MATS * 2 + h) * 1024, at(h));
      }
    }
  };
  float scale = 0.f;  // of token r16
  if constexpr (QUANTIZE) {
    constexpr int HOLD = FEW_CODES / 8 / THREADS;
    const int per = (int)(a.pitch / 8), all = (int)a.M * per;
    typename Vec8<X>::V v[HOLD];
    int left[HOLD], of[HOLD];
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
      const int g = j * THREADS + t, c = g % per * 8;
      of[j] = g < all ? g / per : -1;
      left[j] = g < all ? (a.K - c < 8 ? (int)(a.K - c) : 8) : 0;
      v[j] = {};
      if (left[j] > 0) v[j] = load8(static_cast<const X*>(a.x) + of[j] * a.ldx + c, left[j]);
    }
    if (t < 4) most[t] = 0;
    fetch(s0, wave);
    fetch(s1, wave + WAVES);
    lds_meet();
#pragma unroll
    for (int j = 0; j < HOLD; ++j)
      if (of[j] >= 0) atomicMax(&most[of[j]], magnitude8(widen8<X>(v[j])));
    lds_meet();
    auto scale_of = [&](int r) { return most[r] < 0x7f800000u ? __uint_as_float(most[r]) / 127.f : NAN; };
#pragma unroll
    for (int j = 0; j < HOLD; ++j)
      if (of[j] >= 0) {
        const float s = scale_of(of[j]);
        *reinterpret_cast<unsigned long long*>(codes + (j * THREADS + t) * 8) = !(s > 0.f) ? 0ull : codes8(widen8<X>(v[j]), s, left[j]);
      }
    if (r16 < 4) scale = scale_of(r16);
    lds_meet();
  } else {
    fetch(s0, wave);
    fetch(s1, wave + WAVES);
  }
  i32x4 acc[MATS][TT];
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  const JZ_LDS unsigned char* const mine = (const JZ_LDS unsigned char*)codes + (r16 < a.M ? r16 : 0) * a.pitch;  // other tokens' results are not stored
  auto turn = [&](unsigned char* s, int j) {
    __builtin_amdgcn_sched_barrier(0);
    wait_vmcnt<CH * 2 * (MATS + FROM_X)>();  // this place has landed; the other one's loads were asked for later
    __builtin_amdgcn_sched_barrier(0);
    const JZ_LDS unsigned char* from = (const JZ_LDS unsigned char*)s + wave * PLACE + r16 * 128;
    i32x4 w[CH][2][MATS], x[CH][2][TT];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int at = c * PIECE + (((u * 4 + (lane >> 4)) ^ ((lane >> 1) & 7)) * 16);
#pragma unroll
        for (int i = 0; i < MATS; ++i) w[c][u][i] = *reinterpret_cast<const JZ_LDS i32x4*>(from + at + i * 2048);
        if constexpr (QUANTIZE) {
          const int64_t k = ((int64_t)j * CH + c) * 128 + u * 64 + (lane >> 4) * 16;
          x[c][u][0] = *reinterpret_cast<const JZ_LDS i32x4*>(mine + (k < a.pitch ? k : 0));  // behind the end the weights are zeros
        } else {
#pragma unroll
          for (int k = 0; k < TT; ++k) x[c][u][k] = *reinterpret_cast<const JZ_LDS i32x4*>(from + at + (MATS + k) * 2048);
        }
      }
    __builtin_amdgcn_sched_barrier(0);
    lds_wait<0>();  // read, before the place is filled again
    __builtin_amdgcn_sched_barrier(0);
    fetch(s, j + 2 * WAVES);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < MATS; ++i)
#pragma unroll
          for (int k = 0; k < TT; ++k) acc[i][k] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[c][u][i], x[c][u][k], acc[i][k], 0, 0, 0);
  };
  for (int j = wave; j < places; j += 2 * WAVES) {
    turn(s0, j);
    turn(s1, j + WAVES);  // behind the end: zeros
  }
  wait_vmcnt<0>();
  __syncthreads();  // nothing is on its way into LDS any more
  static_assert(MATS * TT * 1024 <= PLACE, "the sums take a place's room");
  JZ_LDS i32x4* const sums = (JZ_LDS i32x4*)s0;
#pragma unroll
  for (int i = 0; i < MATS; ++i)
#pragma unroll
    for (int j = 0; j < TT; ++j) sums[((wave * MATS + i) * TT + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int s = t; s < TT * 64; s += THREADS) {  // one lane a token and four channels
    const int j = s >> 6, l = s & 63;
    i32x4 v[MATS];
#pragma unroll
    for (int i = 0; i < MATS; ++i) {
      v[i] = sums[(i * TT + j) * 64 + l];
#pragma unroll 4
      for (int q = 1; q < WAVES; ++q) v[i] += sums[((q * MATS + i) * TT + j) * 64 + l];
    }
    const int64_t m = j * 16 + (l & 15);
    if (m >= a.M) continue;
    const float r = QUANTIZE ? scale : a.sx[m];  // s & 15 == lane & 15
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t col = n0 + (l >> 4) * 4 + e;
      if (col >= a.N) break;
      const float f = (float)v[0][e] * (r * a.sw[0][col]);
      if constexpr (GLU) static_cast<Y*>(a.y)[m * a.ldy + col] = (Y)(act_fwd(a.act, f) * ((float)v[MATS - 1][e] * (r * a.sw[MATS - 1][col])));
      else static_cast<Y*>(a.y)[m * a.ldy + col] = (Y)f;
    }
  }
}
