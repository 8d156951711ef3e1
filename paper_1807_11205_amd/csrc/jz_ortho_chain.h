// The steps between A = X X^T and P X (ortho_steps) for matrices whose shorter side is at most 128: a workgroup a matrix, all of a phase's products in one launch.  Included inside
// jz_ortho.hip's anonymous namespace.
//
// Such a product is a microsecond's work, but as a launch of its own takes five: what the launch before wrote has to come back from memory.  Here A and B of a step stay in LDS, in parts as
// everywhere: 128 rows of 512 bytes, 16-byte chunk c of a row at c ^ (row % 16), so that the operands' reads of 16 bytes from 32 rows meet on no bank.  (The writes of 8 bytes do: rows r and r + 16
// have the same banks there; 21.6 % of the LDS cycles are conflicts.)  P, the third matrix, is an operand once a step
// and lies in the workspace.  X X^T itself is a launch before, several workgroups to a tile where X is long: they leave sums in FP32.  Eight wavefronts in 2 x 4, each 64 x 32 of the result;
// symmetric results are computed whole, since storing a tile twice would cost what its products save.
// 128 x 128: 3.5 us a product, of which the matrix instructions and the reads of LDS, 48 each a wavefront, take 1.5 side by side, the results' way through the registers and LDS and
// four barriers a step the rest.  (Sixteen wavefronts of 32 x 32 spill; reads placed among the products by hand change nothing.)
#pragma once

constexpr int CHAIN_SIDE = 128;
struct ChainArgs {
  const float* a;  // [matrix][splits][side][side]: A as the sums that share its product left it, in FP32
  Parts p[2];      // the last P: p[(steps - 1) % 2]
  int splits, steps;
  float ca, cb, cc, shrink;
  const int* skip;
};

template <int KT>  // the padded side / 32
__global__ __launch_bounds__(512, 2) void ortho_chain(ChainArgs a) {
  constexpr int SIDE = 32 * KT, ROW = 512;
  __shared__ __attribute__((aligned(1024))) unsigned char s0[CHAIN_SIDE * ROW], s1[CHAIN_SIDE * ROW];
  if (a.skip && *a.skip) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 2, wn = wave & 3, r32 = lane & 31, half = lane >> 5;
  const int64_t of = blockIdx.x;
  const bool busy = wm * 64 < SIDE && wn * 32 < SIDE;
  auto at = [](int row, int chunk) { return row * ROW + ((chunk ^ (row & 15)) * 16); };
  const float* const from = a.a + of * a.splits * (SIDE * SIDE);
  for (int i = t; i < SIDE * SIDE / 8; i += 512) {
    const int row = i / (SIDE / 8), c = i % (SIDE / 8);
    f32x8 v = load8(from + i * 8);
#pragma unroll 4
    for (int s = 1; s < a.splits; ++s) v += load8(from + s * (SIDE * SIDE) + i * 8);
    const f16x8 hi = __builtin_convertvector(v, f16x8), lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x8), f16x8);
    JZ_LDS unsigned char* const l = (JZ_LDS unsigned char*)s0;
    *reinterpret_cast<JZ_LDS f16x8*>(l + at(row, c / 4 * 8 + c % 4)) = hi;
    *reinterpret_cast<JZ_LDS f16x8*>(l + at(row, c / 4 * 8 + c % 4 + 4)) = lo;
  }
  __syncthreads();
  typedef mm_f32x16 Sum;
  struct Rows {  // an operand's 32 rows: high and low parts of 16 k
    f16x8 hi, lo;
  };
  auto read = [&](const unsigned char* s, int row0, int j) {  // j: which 16 k
    const int c = (j >> 1) * 8 + (j & 1) * 2 + half;
    const JZ_LDS unsigned char* const l = (const JZ_LDS unsigned char*)s;
    return Rows{*reinterpret_cast<const JZ_LDS f16x8*>(l + at(row0 + r32, c)), *reinterpret_cast<const JZ_LDS f16x8*>(l + at(row0 + r32, c + 4))};
  };
  auto add = [](const Rows& x, const Rows& y, Sum& s) {
    s = ElemSplit::mfma(y.hi, x.hi, s);
    s = ElemSplit::mfma(y.hi, x.lo, s);
    s = ElemSplit::mfma(y.lo, x.hi, s);
  };
  auto product = [&](const unsigned char* p, const unsigned char* q, Sum (&s)[2]) {
    s[0] = s[1] = Sum{};
    if (!busy) return;
#pragma unroll
    for (int j = 0; j < 2 * KT; ++j) {
      const Rows y = read(q, wn * 32, j), x0 = read(p, wm * 64, j), x1 = read(p, wm * 64 + 32, j);
      add(x0, y, s[0]);
      add(x1, y, s[1]);
    }
  };
  // f(row, column, four values) for every four columns that a lane has
  auto each = [&](Sum (&s)[2], auto&& f) {
    if (!busy) return;
    static_for<0, 8>([&](auto I) {
      constexpr int x = decltype(I)::value / 4, j = decltype(I)::value % 4;
      f32x4 v = {s[x][4 * j], s[x][4 * j + 1], s[x][4 * j + 2], s[x][4 * j + 3]};
      const int row = wm * 64 + x * 32 + r32;
      if (row < SIDE) f(row, wn * 32 + 8 * j + 4 * half, v);
    });
  };
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  auto split = [](f32x4 v, f16x4* hi, f16x4* lo) {
    *hi = __builtin_convertvector(v, f16x4);
    *lo = __builtin_convertvector(v - __builtin_convertvector(*hi, f32x4), f16x4);
  };
  auto keep = [&](unsigned char* s, int row, int col, f32x4 v) {
    f16x4 hi, lo;
    split(v, &hi, &lo);
    const int c = (col >> 5) * 8 + (col & 31) / 8;
    JZ_LDS unsigned char* const l = (JZ_LDS unsigned char*)s + (col & 4) * 2;
    *reinterpret_cast<JZ_LDS f16x4*>(l + at(row, c)) = hi;
    *reinterpret_cast<JZ_LDS f16x4*>(l + at(row, c + 4)) = lo;
  };
  auto store = [&](const Parts& to, int row, int col, f32x4 v) {
    f16x4 hi, lo;
    split(v, &hi, &lo);
    char* const p = to.row(of, row) + (col >> 5) * 128 + (col & 31) * 2;
    *reinterpret_cast<f16x4*>(p) = hi;
    *reinterpret_cast<f16x4*>(p + 64) = lo;
  };
  Sum s[2];
  for (int i = 0; i < a.steps; ++i) {  // s0: A
    product(s0, s0, s);
    each(s, [&](int row, int col, f32x4 v) {
      const int c = (col >> 5) * 8 + (col & 31) / 8;
      const JZ_LDS unsigned char* const l = (const JZ_LDS unsigned char*)s0 + (col & 4) * 2;
      const f32x4 u = __builtin_convertvector(*reinterpret_cast<const JZ_LDS f16x4*>(l + at(row, c)), f32x4) + __builtin_convertvector(*reinterpret_cast<const JZ_LDS f16x4*>(l + at(row, c + 4)), f32x4);
      f32x4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = fmaf(a.cc / SCALE, v[e], fmaf(a.cb, u[e], row == col + e ? a.ca * SCALE : 0.f));
      keep(s1, row, col, b);
      if (i == 0) store(a.p[0], row, col, b);
    });
    if (i == 0 && a.steps == 1) return;
    __syncthreads();  // s1: B
    if (i > 0) {      // P <- B P, from one place in the workspace to the other
      const char* const p = a.p[(i - 1) & 1].row(of, wn * 32 + r32 < SIDE ? wn * 32 + r32 : 0);
      s[0] = s[1] = Sum{};
      if (busy) {
        Rows y[2 * KT];
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j) {
          const char* const k = p + (j >> 1) * 128 + ((j & 1) * 2 + half) * 16;
          y[j] = Rows{*reinterpret_cast<const f16x8*>(k), *reinterpret_cast<const f16x8*>(k + 64)};
        }
#pragma unroll
        for (int j = 0; j < 2 * KT; ++j) {
          add(read(s1, wm * 64, j), y[j], s[0]);
          add(read(s1, wm * 64 + 32, j), y[j], s[1]);
        }
      }
      each(s, [&](int row, int col, f32x4 v) { store(a.p[i & 1], row, col, v * (a.shrink / SCALE)); });
    }
    if (i + 1 == a.steps) return;
    // A <- B A B
    product(s1, s0, s);
    __syncthreads();
    each(s, [&](int row, int col, f32x4 v) { keep(s0, row, col, v * (1.f / SCALE)); });
    __syncthreads();
    product(s0, s1, s);
    __syncthreads();
    each(s, [&](int row, int col, f32x4 v) { keep(s0, row, col, v * (1.f / SCALE)); });
    __syncthreads();
  }
}

inline int ortho_chain_launch(const ChainArgs& a, int64_t count, hipStream_t st) {
  const unsigned grid = (unsigned)count;
  switch (a.p[0].rows / 32) {
    case 1: ortho_chain<1><<<grid, 512, 0, st>>>(a); break;
    case 2: ortho_chain<2><<<grid, 512, 0, st>>>(a); break;
    case 3: ortho_chain<3><<<grid, 512, 0, st>>>(a); break;
    default: ortho_chain<4><<<grid, 512, 0, st>>>(a); break;
  }
  return jz::launch_status();
}
