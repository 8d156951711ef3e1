// The matrix products of the gated feed-forward block: C[m][n] = sum over k of A(m, k) B(n, k), FP16 or BF16 operands, FP32 sums,
// with the block's activation, product and their derivatives in the epilogue.  Included inside jz_ffn.hip's anonymous namespace.
//
// An operand is k-contiguous (KC, [row][k]) or row-contiguous (MC, [k][row]):
//     forward   gate, up   A = x  KC     B = W_gate and W_up, interleaved 32 rows by 32 rows   KC
//               down       A = h  KC     B = W_down KC
//     backward  dh         A = dy KC     B = W_down MC
//               dx         A = dgate, then dup KC     B = W_gate, then W_up MC         (one sum over 2 F)
//               dW         A = dgate, dup, dy MC      B = x, x, h MC                    (three products in one launch)
//
// Bound: the matrix instructions, that is the clock the card keeps under them (1.5 to 1.8 GHz; they are busy 54 to 70 % of it), with enough rows; with few
// rows or features the tiles that the chip has at a time, and the memory where those are few.  Measured, silu: 16384 rows, 4096 -> 12288 -> 4096 forward
// 1.16 to 1.24 PFLOP/s in BF16 (cards differ); FP16, 8192 rows, 2048 -> 5632 -> 2048 forward and backward, 1.02 to 1.05.
//
// Roundings.  Sums are FP32; h is made from the unrounded gate and up.  What one call leaves for another is in the storage type, as every forward and
// backward tensor is: gate and up, and dgate and dup, which the matrix instructions take in 16 bits anyway.  A weight gradient and
// dx have four such roundings behind them (up, gate through the slope, dgate or dup, their own store; relative 2^-12 each in FP16) instead of the last alone: against 64 bits
// 1.8 to 1.9 times the error of one.  y has two (h and its own), 1.4 times.  In 16 bits h, dgate and dup are what the matrix instructions take; gate and up are a choice: in FP32
// they would double what the forward pass leaves, and making them again backward would add two products to the nine of a training step.
//
// Tiles.  256 x 256 x 64 by eight wavefronts in 2 x 4, each 128 x 64, one workgroup a compute unit; 128 x 128 x 64 by four in 2 x 2, each 64 x 64, two a compute
// unit, where there are too few of the others (jz_ffn.hip: choose).  (256 x 256 by four wavefronts of 128 x 128: 8 % slower, no registers left for reads ahead.)
// 32x32x16 matrix instructions with the operands exchanged, so that a lane has four consecutive n of one m.  Two tiles of operands in LDS:
//     KC  [row][8 chunks of 16 bytes], chunk c at position c ^ (row / 2 % 8); an operand is one 16-byte read (16 lanes at a time reach 256 bytes of
//         banks, two rows: c ^ (row % 8) left every read with a conflict)
//     MC  [k][ROWS / 8 chunks], chunk c at position c ^ 4 (k % 4); an operand is two 8-byte transposing reads
// Both orders keep the reads of a wavefront on different banks.
#pragma once

#include "jz_tile_schedule.h"

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T>
using Op8 = typename Vec8<T>::V;

__device__ __forceinline__ f32x16 mfma(Op8<_Float16> a, Op8<_Float16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(Op8<__bf16> a, Op8<__bf16> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

constexpr int BK = 64;

// ---- activations ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }
constexpr float GELU_K = 0.7978845608028654f, GELU_C = 0.044715f;  // sqrt(2 / pi)

// Phi, the normal distribution function, and bell(v) = exp(-v^2 / 2).  Phi(-|v|) = bell(v) t P(t) with t = 1 / (1 + 0.35 |v|): the factor of the bell is smooth and falls like
// 1 / |v|, and P, of degree 8, was fitted to it for the least
// largest relative error, 7.7e-8 with the coefficients rounded to FP32, up to |v| = 14; with the exponent's rounding the result is within 10 (1 + |v|) 2^-24 of
// itself.  One exponential serves the slope too.  (By erfcf a training pass over 8192 rows, 2048 -> 5632 features took 6 % longer.)
__device__ __forceinline__ float normal(float v, float* bell) {
  constexpr float P[9] = {0.139621407f, 0.139861897f, 0.119832709f, 0.105508648f, -0.0231113750f, 0.159176439f, -0.255716264f, 0.143972680f, -0.0291461349f};
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(v), 0.35f, 1.f));
  float p = P[8];
#pragma unroll
  for (int i = 7; i >= 0; --i) p = fmaf(p, t, P[i]);
  *bell = __builtin_amdgcn_exp2f(v * v * -0.72134752f);  // log2(e) / 2
  const float tail = t * p * *bell;
  return v < 0.f ? tail : 1.f - tail;
}

__device__ __forceinline__ float act_fwd(int kind, float g) {
  if (kind == JZ_ACT_SILU) return g * sigmoid(g);
  if (kind == JZ_ACT_GELU_TANH) return g * sigmoid(2.f * GELU_K * (g + GELU_C * g * g * g));  // (1 + tanh z) / 2 = sigmoid(2 z)
  if (kind == JZ_ACT_GELU) {
    float bell;
    return g * normal(g, &bell);
  }
  return !(g <= 0.f) ? g : 0.f;
}
// act and its derivative
__device__ __forceinline__ float act_both(int kind, float g, float* slope) {
  if (kind == JZ_ACT_SILU) {
    const float s = sigmoid(g);
    *slope = s * (1.f + g * (1.f - s));
    return g * s;
  }
  if (kind == JZ_ACT_GELU_TANH) {
    const float s = sigmoid(2.f * GELU_K * (g + GELU_C * g * g * g));
    // beyond 30 the derivative is 0 or 1 to the last bit, and the cube below may overflow
    *slope = fabsf(g) > 30.f ? (g > 0.f ? 1.f : 0.f) : s + g * s * (1.f - s) * (2.f * GELU_K) * (1.f + 3.f * GELU_C * g * g);
    return g * s;
  }
  if (kind == JZ_ACT_GELU) {
    float bell;
    const float phi = normal(g, &bell);
    *slope = phi + g * bell * 0.3989422804014327f;  // 1 / sqrt(2 pi)
    return g * phi;
  }
  *slope = !(g <= 0.f) ? 1.f : 0.f;
  return !(g <= 0.f) ? g : 0.f;
}

// ---- arguments ------------------------------------------------------------------------------------------------------------
enum { EPI_STORE = 0, EPI_GLU = 1, EPI_GLU_BWD = 2 };

struct Product {           // one product of a launch
  const void *a[2], *b[2];  // [1]: the second part of the sum (dx), or the matrix interleaved with b[0] (gate and up)
  void* c;
  int64_t lda, ldb, ldc;    // elements
  int64_t M, N, K;          // K of one part; N: columns of C (hidden units where gate and up are interleaved)
  int64_t k_rows;           // the rows of an MC operand: K, or less where a KC operand's rows end in zeros that K counts
  bool eights;              // MC operands' rows can be read to a multiple of 8 elements, whatever M and N are
  int tiles_m, tiles_n;
};
struct GemmArgs {
  Product p[3];
  int products, parts;      // parts of the sum: 1 or 2
  int act;
  int full;                 // tiles that one workgroup computes; of each further one `splits` workgroups take tiles_per_split k tiles
  int splits, tiles_per_split;
  unsigned workgroups, first;  // of the product; the first of this launch's
  float* partial;           // [tiles behind `full`][splits][BM][BN]
  const void *gate, *up;    // EPI_GLU_BWD: the saved projections, [M][N]
  void *out0, *out1;        // EPI_GLU: gate and up, or NULL; EPI_GLU_BWD: dgate and dup
  void* padded;             // EPI_GLU: h once more, rows of ld_padded elements that end in zeros, or NULL
  int64_t ld_padded;
};

// dgate and dup of eight elements from dh = v
__device__ __forceinline__ void glu_bwd8(int act, f32x8 v, f32x8 g, f32x8 u, f32x8* dg, f32x8* du) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float slope;
    (*du)[i] = v[i] * act_both(act, g[i], &slope);
    (*dg)[i] = v[i] * u[i] * slope;
  }
}

// ---- results --------------------------------------------------------------------------------------------------------------
// dgate and dup, and where its own rows are not on 16 bytes a second h, lie in the workspace, rows a multiple of 8 long and zero behind their end: they are
// operands of the next products
template <class T>
__device__ __forceinline__ void store_padded(T* p, f32x8 v, int left) {
#pragma unroll
  for (int i = 1; i < 8; ++i) v[i] = i < left ? v[i] : 0.f;
  store8(p, narrow8<T>(v));
}

// What becomes of eight sums (or gate and up sums) that belong to columns n .. n + 7 of row m.
template <class T, int EPI>
__device__ __forceinline__ void finish8(const GemmArgs& a, const Product& p, int64_t m, int64_t n, f32x8 v, f32x8 w) {
  const int left = p.N - n < 8 ? (int)(p.N - n) : 8;
  if (m >= p.M || left <= 0) return;
  if constexpr (EPI == EPI_STORE) {
    store8(static_cast<T*>(p.c) + m * p.ldc + n, narrow8<T>(v), left);
  } else if constexpr (EPI == EPI_GLU) {
    f32x8 h;
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = act_fwd(a.act, v[i]) * w[i];
    store8(static_cast<T*>(p.c) + m * p.ldc + n, narrow8<T>(h), left);
    if (a.padded) store_padded<T>(static_cast<T*>(a.padded) + m * a.ld_padded + n, h, left);
    if (a.out0) {
      store8(static_cast<T*>(a.out0) + m * p.N + n, narrow8<T>(v), left);
      store8(static_cast<T*>(a.out1) + m * p.N + n, narrow8<T>(w), left);
    }
  } else {
    f32x8 dg, du;
    glu_bwd8(a.act, v, widen8<T>(load8(static_cast<const T*>(a.gate) + m * p.N + n, left)), widen8<T>(load8(static_cast<const T*>(a.up) + m * p.N + n, left)), &dg, &du);
    store_padded<T>(static_cast<T*>(a.out0) + m * p.ldc + n, dg, left);
    store_padded<T>(static_cast<T*>(a.out1) + m * p.ldc + n, du, left);
  }
}

// ---- the tile kernel --------------------------------------------------------------------------------------------------------
// One tile of one operand: where a thread's 16-byte chunks come from and go to.
template <class T, bool KC, int ROWS, int THREADS>
struct Staged {
  static constexpr int BYTES = ROWS * BK * 2, CHUNKS = BYTES / 16, EACH = CHUNKS / THREADS;  // chunks a thread
  // chunk i of thread t lies at LDS position (i * THREADS + t) * 16, linear: what an LDS-direct load of a wavefront writes
  static __device__ __forceinline__ void place(int i, int t, int* row, int* k) {
    const int s = i * THREADS + t;
    if constexpr (KC) {
      *row = s >> 3;
      *k = ((s & 7) ^ ((*row >> 1) & 7)) * 8;
    } else {
      constexpr int PER = ROWS / 8;
      *k = s / PER;
      *row = ((s % PER) ^ (4 * (*k & 3))) * 8;
    }
  }
  // Operand x of step s: rows row0 + 32 x .. + 31, k 16 s .. 16 s + 15; lane l has row l % 32, k 8 (l / 32) .. + 7 of the step.  address() gives the four
  // LDS offsets that a lane needs for all of them: KC one a step (an operand is 32 rows = 4 KB further), MC one an operand (a step is 16 k further).
  static __device__ __forceinline__ void address(unsigned (&at)[4], int row0, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (KC) {
        at[i] = (row0 + (lane & 31)) * 128 + (((i * 2 + (lane >> 5)) ^ ((lane >> 1) & 7)) * 16);
      } else {
        // 16 lanes read four k of 16 rows, 8 bytes a lane, and get them transposed: lane i four k of row i
        const int gi = lane >> 4, j = (lane >> 2) & 3, c4 = lane & 3, c = (row0 + 32 * i + 16 * (gi & 1) + 4 * c4) / 8;
        at[i] = (8 * (gi >> 1) + j) * (ROWS * 2) + ((c ^ (4 * j)) * 16) + (c4 & 1) * 8;
      }
    }
  }
  static __device__ __forceinline__ Op8<T> read(const JZ_LDS unsigned char* lds, const unsigned (&at)[4], int x, int s) {
    if constexpr (KC) {
      return *reinterpret_cast<const JZ_LDS Op8<T>*>(lds + at[s] + x * 4096);
    } else {
      struct { s16x4 lo, hi; } v;
      v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((JZ_LDS s16x4*)(lds + at[x] + s * (16 * ROWS * 2)));
      v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((JZ_LDS s16x4*)(lds + at[x] + s * (16 * ROWS * 2) + 4 * (ROWS * 2)));
      return __builtin_bit_cast(Op8<T>, v);
    }
  }
};

// Which tile of which product a workgroup has.  Consecutive workgroups land on different XCDs, each with an L2 of its own, so every XCD gets a run of
// tiles, and within a run four rows of tiles are taken column by column: what a run reads at a time is then a block.  (Eight and sixteen rows: within 2 %.)
struct Tile {
  int product, split;  // split < 0: the whole sum
  unsigned m, n, behind;  // behind: number among the tiles that are split
};
__device__ __forceinline__ void place_tile(const GemmArgs& a, unsigned t, Tile* w) {
  w->product = 0;
  while (w->product + 1 < a.products && t >= (unsigned)(a.p[w->product].tiles_m * a.p[w->product].tiles_n)) {
    t -= a.p[w->product].tiles_m * a.p[w->product].tiles_n;
    ++w->product;
  }
  const unsigned rows = a.p[w->product].tiles_m, cols = a.p[w->product].tiles_n, G = 4;
  const unsigned band = t / (G * cols), in = t % (G * cols), high = rows - band * G < G ? rows - band * G : G;
  w->m = band * G + in % high;
  w->n = in / high;
}
__device__ __forceinline__ Tile find_tile(const GemmArgs& a) {
  Tile w;
  const unsigned full = a.full, number = a.first + blockIdx.x;
  if (number < full) {
    w.split = -1;
    w.behind = 0;
    place_tile(a, xcd_remap(number, full), &w);
  } else {
    const unsigned i = number - full, rest = (a.workgroups - full) / a.splits;
    w.split = i / rest;
    w.behind = i % rest;
    place_tile(a, full + w.behind, &w);
  }
  return w;
}

// The sums of a wavefront's tile to their places: FP32 partial sums, or the epilogue.  They pass through LDS 32 rows at a time, so that a lane has eight columns
// of a row and neighbouring lanes its neighbours: whole lines are stored.  lds: 32 rows of TN * 32 floats of the wavefront's own, 16-byte chunk c of row r at
// c ^ (r % 16).  Register 4 j + i of a lane holds row lane % 32, column 8 j + 4 (lane / 32) + i.
// partial: where the sums of the wavefront's first row and column go instead, rows `pitch` apart; or NULL.
template <class T, int EPI, int TM, int TN>
__device__ __forceinline__ void finish_tile(const GemmArgs& a, const Product& p, f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, float* partial, int pitch,
                                            JZ_LDS unsigned char* lds, int lane) {
  static_assert(TN % 2 == 0, "16 chunks or more a row");
  constexpr int PITCH = TN * 128, PER = (EPI == EPI_GLU ? TN * 2 : TN * 4);  // bytes of a row; groups of eight results in one
  auto chunk = [&](int row, int c) { return lds + row * PITCH + ((c ^ (row & 15)) * 16); };
  auto eight = [&](int row, int c) {
    const f32x4 lo = *reinterpret_cast<const JZ_LDS f32x4*>(chunk(row, c)), hi = *reinterpret_cast<const JZ_LDS f32x4*>(chunk(row, c + 1));
    return f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  };
  static_for<0, TM>([&](auto X) {
    constexpr int x = decltype(X)::value;
    static_for<0, TN * 4>([&](auto I) {
      constexpr int y = decltype(I)::value / 4, j = decltype(I)::value % 4;
      *reinterpret_cast<JZ_LDS f32x4*>(chunk(lane & 31, y * 8 + j * 2 + (lane >> 5))) = f32x4{acc[x][y][4 * j], acc[x][y][4 * j + 1], acc[x][y][4 * j + 2], acc[x][y][4 * j + 3]};
    });
    if (partial) {
#pragma unroll 1
      for (int i = lane; i < 32 * TN * 4; i += 64) {
        const int row = i / (TN * 4), c = i % (TN * 4);
        store8(partial + (x * 32 + row) * pitch + c * 8, eight(row, c * 2));
      }
    } else {
#pragma unroll 1
      for (int i = lane; i < 32 * PER; i += 64) {
        const int row = i / PER, c = i % PER;
        if constexpr (EPI == EPI_GLU) {  // gate and up alternate by 32 columns
          const int g = (c >> 2) * 16 + (c & 3) * 2;
          finish8<T, EPI>(a, p, m0 + x * 32 + row, n0 / 2 + c * 8, eight(row, g), eight(row, g + 8));
        } else {
          const f32x8 v = eight(row, c * 2);
          finish8<T, EPI>(a, p, m0 + x * 32 + row, n0 + c * 8, v, v);
        }
      }
    }
  });
}

// The same for EPI_GLU_BWD, whose results need gate and up from memory: those of a strip are asked for a strip ahead.
template <class T, int ACT, int TM, int TN>
__device__ __forceinline__ void finish_bwd(const GemmArgs& a, const Product& p, f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, JZ_LDS unsigned char* lds, int lane) {
  constexpr int PITCH = TN * 128, PER = TN * 4, EACH = 32 * PER / 64;
  typename Vec8<T>::V g[EACH], u[EACH];
  auto place = [&](int x, int i, int64_t* m, int64_t* n) {
    const int s = i * 64 + lane;
    *m = m0 + x * 32 + s / PER;
    *n = n0 + s % PER * 8;
    return *m < p.M && *n < p.N;
  };
  auto ask = [&](int x, int i) {
    int64_t m, n;
    if (!place(x, i, &m, &n)) return;
    const int64_t at = m * p.N + n;
    const int left = at + 8 > p.M * p.N ? (int)(p.N - n) : 8;  // what follows a row's end is read and not stored; behind the last row there is nothing
    g[i] = load8(static_cast<const T*>(a.gate) + at, left);
    u[i] = load8(static_cast<const T*>(a.up) + at, left);
  };
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    g[i] = u[i] = {};
    ask(0, i);
  }
  auto chunk = [&](int row, int c) { return lds + row * PITCH + ((c ^ (row & 15)) * 16); };
  static_for<0, TM>([&](auto X) {
    constexpr int x = decltype(X)::value;
    static_for<0, TN * 4>([&](auto I) {
      constexpr int y = decltype(I)::value / 4, j = decltype(I)::value % 4;
      *reinterpret_cast<JZ_LDS f32x4*>(chunk(lane & 31, y * 8 + j * 2 + (lane >> 5))) = f32x4{acc[x][y][4 * j], acc[x][y][4 * j + 1], acc[x][y][4 * j + 2], acc[x][y][4 * j + 3]};
    });
    static_for<0, EACH>([&](auto I) {
      constexpr int i = decltype(I)::value;
      const int s = i * 64 + lane, row = s / PER, c = s % PER * 2;
      const f32x4 lo = *reinterpret_cast<const JZ_LDS f32x4*>(chunk(row, c)), hi = *reinterpret_cast<const JZ_LDS f32x4*>(chunk(row, c + 1));
      f32x8 dg, du;
      glu_bwd8(ACT, f32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}, widen8<T>(g[i]), widen8<T>(u[i]), &dg, &du);
      if constexpr (x + 1 < TM) ask(x + 1, i);
      int64_t m, n;
      if (place(x, i, &m, &n)) {
        const int left = p.N - n < 8 ? (int)(p.N - n) : 8;
        store_padded<T>(static_cast<T*>(a.out0) + m * p.ldc + n, dg, left);
        store_padded<T>(static_cast<T*>(a.out1) + m * p.ldc + n, du, left);
      }
    });
  });
}

template <class T, int EPI, int ACT, int TM, int TN>
__device__ __forceinline__ void finish(const GemmArgs& a, const Product& p, f32x16 (&acc)[TM][TN], int64_t m0, int64_t n0, float* partial, int pitch,
                                       JZ_LDS unsigned char* lds, int lane) {
  if constexpr (EPI == EPI_GLU_BWD) {
    if (partial) finish_tile<T, EPI_STORE>(a, p, acc, m0, n0, partial, pitch, lds, lane);
    else finish_bwd<T, ACT>(a, p, acc, m0, n0, lds, lane);
  } else {
    finish_tile<T, EPI>(a, p, acc, m0, n0, partial, pitch, lds, lane);
  }
}

// Any sizes, any alignment, at about half the rate of the LDS-direct kernels: the operands pass through registers on their way into LDS, the next tile's while a tile is multiplied.  Loads are full vectors without
// branches (global memory takes them at any alignment), from where the element is or would be: rows outside are the last row, and what follows a row's end belongs to
// no result, or to the end of the sum, where it is cleared.  Only the vectors that would pass the tensor's last element are loaded one by one.
template <class T, bool KC>
struct AnySource {
  int64_t ld, rows, K;
  __device__ __forceinline__ Op8<T> load(const T* p, int64_t row, int64_t k) const {
    const int64_t r = row < rows ? row : rows - 1, kk = k < K ? k : K - 1, at = KC ? r * ld + kk : kk * ld + r;
    const int64_t all = KC ? (rows - 1) * ld + K : (K - 1) * ld + rows;
    if (at + 8 > all) return load8(p + at, (int)(KC ? K - kk : rows - r));  // less than eight to the row's end then
    return load8(p + at);
  }
  __device__ __forceinline__ Op8<T> cleared(Op8<T> v, int64_t k) const {  // behind the end of the sum
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (KC ? k + e : k) < K ? v[e] : T(0.f);
    return v;
  }
};

// ACT: the activation where EPI is EPI_GLU_BWD, else 0
template <class T, bool KCA, bool KCB, int EPI, int ACT, int BM, int BN>
__global__ __launch_bounds__(256, 2) void ffn_gemm_any(GemmArgs a) {
  using SA = Staged<T, KCA, BM, 256>;
  using SB = Staged<T, KCB, BN, 256>;
  constexpr int TM = BM / 64, TN = BN / 64;
  __shared__ __attribute__((aligned(1024))) unsigned char operands[2][SA::BYTES + SB::BYTES];
  static_assert(SA::BYTES + SB::BYTES >= 4 * 32 * TN * 128, "the results pass through LDS");
  const Tile w = find_tile(a);
  const Product p = a.p[w.product];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 1, wn = wave & 1;
  const int64_t m0 = (int64_t)w.m * BM, n0 = (int64_t)w.n * BN;
  const int per_part = (int)((p.K + BK - 1) / BK), all = per_part * a.parts;
  const int first = w.split < 0 ? 0 : w.split * a.tiles_per_split, last = w.split < 0 || first + a.tiles_per_split > all ? all : first + a.tiles_per_split;
  float* const partial = w.split < 0 ? nullptr : a.partial + ((size_t)w.behind * a.splits + w.split) * (BM * BN);
  const AnySource<T, KCA> from_a = {p.lda, p.M, p.k_rows};
  const AnySource<T, KCB> from_b = {p.ldb, p.N, p.k_rows};

  Op8<T> ra[SA::EACH], rb[SB::EACH];
  auto fetch = [&](int kt) {
    const int part = kt >= per_part;
    const int64_t k0 = (int64_t)(kt - part * per_part) * BK;
#pragma unroll
    for (int i = 0; i < SA::EACH; ++i) {
      int row, k;
      SA::place(i, t, &row, &k);
      ra[i] = from_a.load(static_cast<const T*>(p.a[part]), m0 + row, k0 + k);
    }
#pragma unroll
    for (int i = 0; i < SB::EACH; ++i) {
      int row, k;
      SB::place(i, t, &row, &k);
      if constexpr (EPI == EPI_GLU) rb[i] = from_b.load(static_cast<const T*>((row >> 5) & 1 ? p.b[1] : p.b[0]), n0 / 2 + (row >> 6) * 32 + (row & 31), k0 + k);
      else rb[i] = from_b.load(static_cast<const T*>(p.b[part]), n0 + row, k0 + k);
    }
    if (k0 + BK > p.k_rows) {
#pragma unroll
      for (int i = 0; i < SA::EACH; ++i) {
        int row, k;
        SA::place(i, t, &row, &k);
        ra[i] = from_a.cleared(ra[i], k0 + k);
      }
#pragma unroll
      for (int i = 0; i < SB::EACH; ++i) {
        int row, k;
        SB::place(i, t, &row, &k);
        rb[i] = from_b.cleared(rb[i], k0 + k);
      }
    }
  };
  auto put = [&](unsigned char* lds) {
#pragma unroll
    for (int i = 0; i < SA::EACH; ++i) *reinterpret_cast<Op8<T>*>(lds + (i * 256 + t) * 16) = ra[i];
#pragma unroll
    for (int i = 0; i < SB::EACH; ++i) *reinterpret_cast<Op8<T>*>(lds + SA::BYTES + (i * 256 + t) * 16) = rb[i];
  };
  unsigned at_a[4], at_b[4];
  SA::address(at_a, wm * (BM / 2), lane);
  SB::address(at_b, wn * (BN / 2), lane);
  f32x16 acc[TM][TN];
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y) acc[x][y] = f32x16{};
  if (first < last) {
    fetch(first);
    put(operands[0]);
  }
  __syncthreads();
  for (int kt = first; kt < last; ++kt) {
    const JZ_LDS unsigned char* const lds = (const JZ_LDS unsigned char*)operands[(kt - first) & 1];
    if (kt + 1 < last) fetch(kt + 1);
#pragma unroll
    for (int s = 0; s < BK / 16; ++s) {
      Op8<T> fa[TM], fb[TN];
#pragma unroll
      for (int x = 0; x < TM; ++x) fa[x] = SA::read(lds, at_a, x, s);
#pragma unroll
      for (int y = 0; y < TN; ++y) fb[y] = SB::read(lds + SA::BYTES, at_b, y, s);
#pragma unroll
      for (int x = 0; x < TM; ++x)
#pragma unroll
        for (int y = 0; y < TN; ++y) acc[x][y] = mfma(fb[y], fa[x], acc[x][y]);
    }
    if (kt + 1 < last) put(operands[(kt + 1 - first) & 1]);
    __syncthreads();
  }
  finish<T, EPI, ACT>(a, p, acc, m0 + wm * (BM / 2), n0 + wn * (BN / 2), partial ? partial + wm * (BM / 2) * BN + wn * (BN / 2) : nullptr, BN,
                      (JZ_LDS unsigned char*)operands[0] + wave * (32 * TN * 128), lane);
}

// ---- LDS-direct ---------------------------------------------------------------------------------------------------------------
// Where one operand's tile comes from.
template <class T, bool KC, int ROWS, int THREADS, bool DUAL>
struct Source {
  using S = Staged<T, KC, ROWS, THREADS>;
  const char* base[2];  // of the tile's rows: part 0 and 1 of the sum, or the two interleaved matrices
  int64_t pitch, rows_left, K;
  unsigned off, step;   // of the thread's first chunk, and from one to the next
  int k;                // the chunk's place in a tile: k of KC, for the end of the sum

  __device__ __forceinline__ void init(const void* const* p, int64_t ld, int64_t row0, int64_t rows, int64_t K_, int t) {
    pitch = ld * 2;
    rows_left = (KC ? rows : (rows + 7) & ~int64_t(7)) - row0;  // an MC operand's rows can be read in eights
    K = K_;
    base[0] = static_cast<const char*>(p[0]) + row0 * (KC ? pitch : 2);
    base[1] = static_cast<const char*>(p[1]) + row0 * (KC ? pitch : 2);
    int row;
    S::place(0, t, &row, &k);
    int row1, k1;
    S::place(1, t, &row1, &k1);
    step = KC ? (unsigned)((DUAL ? 32 : row1 - row) * pitch) : (unsigned)((k1 - k) * pitch);
    if (DUAL) row &= 31;
    off = KC ? (unsigned)(row * pitch + k * 2) : (unsigned)(k * pitch + row * 2);
  }
  // 16 bytes a lane into LDS; what lies outside the operand arrives as zeros
  template <class L>
  __device__ __forceinline__ void load(L* lds, int part, int64_t k0, int wave, bool wanted) const {
    const int64_t skip = wanted ? k0 * (KC ? 2 : pitch) : 0;
    const int64_t span = KC ? (rows_left - 1) * pitch + (K - k0) * 2 : (K - k0 - 1) * pitch + rows_left * 2;
    const int bytes = !wanted || span < 0 ? 0 : (int)(span < 0x7ffffff0 ? span : 0x7ffffff0);
    const auto r0 = __builtin_amdgcn_make_buffer_rsrc((void*)(base[DUAL ? 0 : part] + skip), 0, bytes, 0x00020000);
    const auto r1 = __builtin_amdgcn_make_buffer_rsrc((void*)(base[1] + skip), 0, bytes, 0x00020000);
    const unsigned end = KC && k >= K - k0 ? 0x80000000u : 0u;  // a row's end inside the tile: the next row does not follow
#pragma unroll
    for (int i = 0; i < S::EACH; ++i) {
      // interleaved by 32 rows: 256 threads bring 32 rows at a time, 512 threads 64
      const bool second = DUAL && (THREADS == 256 ? i & 1 : wave >> 2);
      const unsigned at = (off + (DUAL && THREADS == 256 ? i >> 1 : i) * step) | end;
      jz_dma16(second ? r1 : r0, (lds_byte*)lds + (i * THREADS + wave * 64) * 16, at);
    }
  }
};

template <class T, bool KCA, bool KCB, int EPI, int ACT, int BM, int BN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN, 2) void ffn_gemm(GemmArgs a) {
  constexpr int THREADS = 64 * WGM * WGN, TM = BM / WGM / 32, TN = BN / WGN / 32, STEPS = BK / 16, READS = TM * (KCA ? 1 : 2) + TN * (KCB ? 1 : 2);
  using SA = Staged<T, KCA, BM, THREADS>;
  using SB = Staged<T, KCB, BN, THREADS>;
  // four objects, not one: an LDS read then only waits for the loads into its own
  __shared__ __attribute__((aligned(1024))) unsigned char a0[SA::BYTES], a1[SA::BYTES], b0[SB::BYTES], b1[SB::BYTES];
  const Tile w = find_tile(a);
  const Product p = a.p[w.product];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WGN, wn = wave % WGN;
  const int64_t m0 = (int64_t)w.m * BM, n0 = (int64_t)w.n * BN;
  const int per_part = (int)((p.K + BK - 1) / BK), all = per_part * a.parts;
  const int first = w.split < 0 ? 0 : w.split * a.tiles_per_split, last = w.split < 0 || first + a.tiles_per_split > all ? all : first + a.tiles_per_split;
  float* const partial = w.split < 0 ? nullptr : a.partial + ((size_t)w.behind * a.splits + w.split) * (BM * BN);

  Source<T, KCA, BM, THREADS, false> from_a;
  Source<T, KCB, BN, THREADS, EPI == EPI_GLU> from_b;
  from_a.init(p.a, p.lda, m0, p.M, KCA ? p.K : p.k_rows, t);
  from_b.init(p.b, p.ldb, EPI == EPI_GLU ? n0 / 2 : n0, p.N, KCB ? p.K : p.k_rows, t);
  auto fetch = [&](auto* la, auto* lb, int kt) {
    const int part = kt >= per_part && a.parts > 1;  // behind the last tile: zeros, so that there is no branch among the products
    const int64_t k0 = (int64_t)(kt - part * per_part) * BK;
    from_a.load(la, part, k0, wave, kt < last);
    from_b.load(lb, part, k0, wave, kt < last);
  };
  unsigned at_a[4], at_b[4];
  SA::address(at_a, wm * TM * 32, lane);
  SB::address(at_b, wn * TN * 32, lane);
  f32x16 acc[TM][TN];
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y) acc[x][y] = f32x16{};
  Op8<T> fa[2][TM], fb[2][TN];
  auto read = [&](auto* la, auto* lb, int s, int to) {
#pragma unroll
    for (int x = 0; x < TM; ++x) fa[to][x] = SA::read((const JZ_LDS unsigned char*)la, at_a, x, s);
#pragma unroll
    for (int y = 0; y < TN; ++y) fb[to][y] = SB::read((const JZ_LDS unsigned char*)lb, at_b, y, s);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y) acc[x][y] = mfma(fb[from][y], fa[from][x], acc[x][y]);
  };
  // The tile in la, lb.  The products of its predecessor's last step run while its first operands are read and the next tile is asked for, into the place
  // that the predecessor leaves.  The loop turns at the barrier: loads that are in flight across its turn would be waited for.
  auto tile = [&](auto* la, auto* lb, auto* na, auto* nb, int kt) {
    all_landed();
    read(la, lb, 0, 0);
    fetch(na, nb, kt + 1);
    multiply((STEPS - 1) & 1);
    spread_out<TM * TN, READS, SA::EACH + SB::EACH>();
    static_for<0, STEPS - 1>([&](auto S) {
      constexpr int s = decltype(S)::value;
      read(la, lb, s + 1, (s + 1) & 1);
      multiply(s & 1);
      spread_out<TM * TN, READS, 0>();
    });
  };
  if (first < last) {
#pragma unroll
    for (int x = 0; x < TM; ++x) fa[1][x] = Op8<T>{};  // the first tile has no predecessor
#pragma unroll
    for (int y = 0; y < TN; ++y) fb[1][y] = Op8<T>{};
    fetch(a0, b0, first);
    for (int kt = first; kt < last; kt += 2) {
      tile(a0, b0, a1, b1, kt);
      if (kt + 1 < last) tile(a1, b1, a0, b0, kt + 1);
    }
    multiply((STEPS - 1) & 1);
  }
  all_landed();  // zeros too: the results take the operands' place
  constexpr int STRIP = 32 * TN * 128, FIT = SA::BYTES / STRIP;
  static_assert(2 * FIT >= WGM * WGN, "the results pass through the place of A");
  unsigned char* const mine = (wave < FIT ? a0 + wave * STRIP : a1 + (wave - FIT) * STRIP);
  finish<T, EPI, ACT>(a, p, acc, m0 + wm * TM * 32, n0 + wn * TN * 32, partial ? partial + wm * TM * 32 * BN + wn * TN * 32 : nullptr, BN, (JZ_LDS unsigned char*)mine, lane);
}

// The partial sums of the tiles that are split, added in the order of the splits, and the epilogue.  Eight columns a thread, blockIdx.y a tile.
template <class T, int EPI, int TILE>
__global__ __launch_bounds__(256) void ffn_join(GemmArgs a) {
  constexpr int PER = EPI == EPI_GLU ? TILE / 16 : TILE / 8;  // groups of eight results in a row of a tile
  Tile w;
  place_tile(a, a.full + blockIdx.y, &w);
  const Product& p = a.p[w.product];
  const int i = blockIdx.x * 256 + threadIdx.x, row = i / PER, c = i % PER;
  const int64_t m = (int64_t)w.m * TILE + row, n = (int64_t)w.n * (EPI == EPI_GLU ? TILE / 2 : TILE) + c * 8;
  if (m >= p.M || n >= p.N) return;
  auto total = [&](int col) {
    const float* f = a.partial + (size_t)blockIdx.y * a.splits * (TILE * TILE) + row * TILE + col;
    f32x8 v = load8(f);
    for (int s = 1; s < a.splits; ++s) v += load8(f + (size_t)s * (TILE * TILE));
    return v;
  };
  const int col = EPI == EPI_GLU ? (c >> 2) * 64 + (c & 3) * 8 : c * 8;
  const f32x8 v = total(col), u = EPI == EPI_GLU ? total(col + 32) : v;
  finish8<T, EPI>(a, p, m, n, v, u);
}

// Copies of matrices with rows on 16 bytes, zeros behind a row's end, for operands whose rows are not.  Eight elements a thread.
struct Copies {
  struct One {
    const void* from;
    void* to;
    int64_t rows, cols, ld, pitch, first;  // first: its first block
  } m[6];
  int count;
  int64_t first;  // the launch's first block
};
template <class T>
__global__ __launch_bounds__(256) void ffn_copy(Copies c) {
  const int64_t block = c.first + blockIdx.x;
  int q = 0;
  while (q + 1 < c.count && block >= c.m[q + 1].first) ++q;
  const Copies::One& o = c.m[q];
  const int64_t i = (block - o.first) * 256 + threadIdx.x, per = o.pitch / 8, row = i / per, col = (i - row * per) * 8;
  if (row >= o.rows) return;
  const int64_t left = o.cols - col;
  store8(static_cast<T*>(o.to) + row * o.pitch + col, load8(static_cast<const T*>(o.from) + row * o.ld + col, left < 8 ? (int)left : 8));
}
