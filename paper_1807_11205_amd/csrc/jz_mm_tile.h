// Matrix products C[m][n] = sum over k of A[m][k] B[n][k], both operands k-contiguous, whose elements are not plain 16-bit numbers: 8-bit integers (jz_i8.hip), and FP32 values
// as two FP16 parts (jz_ortho.hip).  Included inside a kernel file's anonymous namespace, behind jz_lds_dma.h and jz_tile_schedule.h.
//
// To the loads an operand is rows of bytes.  A tile of it is BM (BN) rows x 128 bytes, brought in by LDS-direct loads, two stages; 16-byte chunk c of a row lies at
// c ^ (row / 2 % 8), so that neither the loads' writes nor the operands' reads meet on a bank.  An operand register is 16 bytes of a row for each lane: lane l has row l % 32 and
// chunk 2 s + l / 32 in step s = 0 .. 3.  Three kinds of elements:
//     ElemI8     128 int8 of k; a step is one 32x32x32 matrix instruction, sums are int32 and exact
//     ElemSplit  32 k of an FP32 value v as hi = FP16(v) (chunks 0-3) and lo = FP16(v - hi) (chunks 4-7), 22 bits together.  A product is hi hi + hi lo + lo hi: three
//                instructions for each two reads of an operand, so that the matrix instructions and not LDS are what the loop waits for
// Bound, 256 x 256: the matrix instructions.  16384 rows 4096 -> 12288 of ElemI8 in 700 us, 2.3 POP/s (the library's product of 8192^3 2.1); ElemSplit, 4096 x 4096 times 4096 x 12288, 914 us,
// 1.35 PFLOP/s of matrix instructions (FP16 library 1.36), which are busy 79 % of 1.6 GHz; 16 products
// of 1024^3 that fill 160 of the compute units 78 us, 20 of them results on their way.
// Sums are in exchanged order (B's rows first): register 4 j + i of a lane holds row lane % 32, column 8 j + 4 (lane / 32) + i.
#pragma once

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float mm_f32x16 __attribute__((ext_vector_type(16)));

struct ElemI8 {
  typedef i32x4 Reg;
  typedef i32x16 Sum;
  typedef int Val;
  static constexpr bool SPLIT = false;
  static __device__ __forceinline__ Sum mfma(Reg a, Reg b, Sum c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0); }
};
struct ElemSplit {
  typedef f16x8 Reg;
  typedef mm_f32x16 Sum;
  typedef float Val;
  static constexpr bool SPLIT = true;
  static __device__ __forceinline__ Sum mfma(Reg a, Reg b, Sum c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

struct MmOperand {
  const void* p[2];        // [1]: the matrix interleaved with [0], 32 rows by 32 rows (B only)
  int64_t rows, pitch, of; // rows of one matrix; bytes from a row to the next and from one matrix of a batch to the next
};
struct MmArgs {
  MmOperand a, b;
  int64_t row_bytes;       // of k: a multiple of 16
  int tiles_m, tiles_n;
  unsigned tiles;          // of one matrix of the batch; in all `workgroups`
  unsigned workgroups, first;
  bool symmetric;          // only tiles on and below the diagonal
  const int* skip;         // or NULL: nothing is done where it is not 0
  int splits;              // mm_tiny: workgroups that share a tile's sum, each with results of its own (w.of counts matrices times splits)
};

// Where a workgroup's tile lies.  Consecutive workgroups land on different XCDs, each with an L2 of its own, so every XCD gets a run of tiles; within it four rows of
// tiles are taken column by column, or the lower triangle row by row.
struct MmTile {
  unsigned of, m, n;
};
__device__ __forceinline__ MmTile mm_tile(const MmArgs& a) {
  unsigned t = xcd_remap(a.first + blockIdx.x, a.workgroups);
  MmTile w;
  w.of = t / a.tiles;
  t -= w.of * a.tiles;
  if (a.symmetric) {
    unsigned m = (unsigned)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while (m * (m + 1) / 2 > t) --m;
    while ((m + 1) * (m + 2) / 2 <= t) ++m;
    w.m = m;
    w.n = t - m * (m + 1) / 2;
  } else {
    const unsigned G = 4, cols = a.tiles_n, band = t / (G * cols), in = t % (G * cols), high = a.tiles_m - band * G < G ? a.tiles_m - band * G : G;
    w.m = band * G + in % high;
    w.n = in / high;
  }
  return w;
}

// One operand's tile: ROWS x 128 bytes by THREADS threads, 16 bytes each at a time.
template <int ROWS, int THREADS, bool DUAL>
struct MmSource {
  static constexpr int BYTES = ROWS * 128, EACH = BYTES / 16 / THREADS;
  static_assert(EACH >= 1 && (!DUAL || THREADS >= 256), "");
  const char* base[2];
  int64_t pitch, rows_left, row_bytes;
  unsigned off, step, chunk;

  __device__ __forceinline__ void init(const MmOperand& o, int64_t of, int64_t row0, int64_t row_bytes_, int t) {
    pitch = o.pitch;
    row_bytes = row_bytes_;
    rows_left = o.rows - row0;
    base[0] = static_cast<const char*>(o.p[0]) + of * o.of + row0 * pitch;
    base[1] = static_cast<const char*>(o.p[DUAL ? 1 : 0]) + of * o.of + row0 * pitch;
    const int row = t >> 3;
    chunk = (((t & 7) ^ ((row >> 1) & 7)) * 16);
    step = (unsigned)((DUAL ? 32 : THREADS / 8) * pitch);
    off = (unsigned)((DUAL ? row & 31 : row) * pitch) + chunk;
  }
  // bytes k0 .. k0 + 127 of the rows into registers
  template <class V>
  __device__ __forceinline__ void get(V (&to)[EACH], int64_t k0, bool wanted) const {
    static_assert(!DUAL, "");
    const int64_t span = (rows_left - 1) * pitch + row_bytes - k0;
    const int bytes = !wanted || span < 0 ? 0 : (int)(span < 0x7ffffff0 ? span : 0x7ffffff0);
    const auto r = __builtin_amdgcn_make_buffer_rsrc((void*)(base[0] + (wanted ? k0 : 0)), 0, bytes, 0x00020000);
    const unsigned end = (int64_t)chunk >= row_bytes - k0 ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < EACH; ++i) to[i] = __builtin_bit_cast(V, __builtin_amdgcn_raw_buffer_load_b128(r, (int)((off + i * step) | end), 0, 0));
  }
  // bytes k0 .. k0 + 127 of the rows into LDS; what lies outside the operand arrives as zeros
  template <class L>
  __device__ __forceinline__ void load(L* lds, int64_t k0, int wave, bool wanted) const {
    const int64_t skip = wanted ? k0 : 0, span = (rows_left - 1) * pitch + row_bytes - k0;
    const int bytes = !wanted || span < 0 ? 0 : (int)(span < 0x7ffffff0 ? span : 0x7ffffff0);
    const auto r0 = __builtin_amdgcn_make_buffer_rsrc((void*)(base[0] + skip), 0, bytes, 0x00020000);
    const auto r1 = __builtin_amdgcn_make_buffer_rsrc((void*)(base[1] + skip), 0, bytes, 0x00020000);
    const unsigned end = (int64_t)chunk >= row_bytes - k0 ? 0x80000000u : 0u;  // a row's end inside the tile
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const bool second = DUAL && (THREADS == 256 ? i & 1 : wave >> 2);  // 256 threads bring 32 rows at a time, 512 threads 64
      const unsigned at = (off + (DUAL && THREADS == 256 ? i >> 1 : i) * step) | end;
      jz_dma16(second ? r1 : r0, (lds_byte*)lds + (i * THREADS + wave * 64) * 16, at);
    }
  }
};

// The sums of 32 rows of a wavefront's tile, in LDS: TN * 32 columns of 32 bits, 16-byte chunk c of row r at c ^ (r % 16) (TN 1: % 8).  put and row8 meet on no bank; col8 does, since rows r and r + 16
// have one order: 11 to 18 % of the LDS cycles of the update's products of 2816 x 1024, 6 % of those of 4096 x 12288, none where a last product stores rows alone.
template <class E, int TN>
struct MmStrip {
  static constexpr int PITCH = TN * 128, MASK = TN > 1 ? 15 : 7, COLS = TN * 32;
  JZ_LDS unsigned char* lds;
  typedef typename E::Val V;
  typedef V V4 __attribute__((ext_vector_type(4)));
  __device__ __forceinline__ JZ_LDS V4* chunk(int row, int c) const { return reinterpret_cast<JZ_LDS V4*>(lds + row * PITCH + ((c ^ (row & MASK)) * 16)); }
  __device__ __forceinline__ void put(const typename E::Sum* s, int lane) const {
    static_for<0, TN * 4>([&](auto I) {
      constexpr int y = decltype(I)::value / 4, j = decltype(I)::value % 4;
      *chunk(lane & 31, y * 8 + j * 2 + (lane >> 5)) = V4{s[y][4 * j], s[y][4 * j + 1], s[y][4 * j + 2], s[y][4 * j + 3]};
    });
  }
  // columns col .. col + 7 of a row
  __device__ __forceinline__ void row8(int row, int col, V (&v)[8]) const {
    const V4 lo = *chunk(row, col / 4), hi = *chunk(row, col / 4 + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lo[i], v[4 + i] = hi[i];
  }
  __device__ __forceinline__ void set_row8(int row, int col, const V (&v)[8]) const {
    *chunk(row, col / 4) = V4{v[0], v[1], v[2], v[3]};
    *chunk(row, col / 4 + 1) = V4{v[4], v[5], v[6], v[7]};
  }
  // rows row .. row + 7 of a column
  __device__ __forceinline__ void col8(int row, int col, V (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = reinterpret_cast<const JZ_LDS V*>(chunk(row + i, col / 4))[col % 4];
  }
};

// epi.strip(strip, tile, m, n, lane): what becomes of rows m .. m + 31 and columns n .. n + COLS - 1 of a matrix; a wavefront with an odd number of sums across (192 x 192) hands them out one by one.
// 192 x 192: four wavefronts with 144 registers of sums each, one on a SIMD; 54 matrix instructions for 24 reads of LDS, a third fewer for each product than 128 x 128 has.
template <class E, class Epi, int BM, int BN, int WGM, int WGN, bool DUAL>
__global__ __launch_bounds__(64 * WGM * WGN, BM == 192 ? 1 : 2) void mm_tiles(MmArgs a, Epi epi) {
  constexpr int THREADS = 64 * WGM * WGN, TM = BM / WGM / 32, TN = BN / WGN / 32, READS = TM + TN;
  typedef typename E::Reg Reg;
  typedef typename E::Sum Sum;
  using SA = MmSource<BM, THREADS, false>;
  using SB = MmSource<BN, THREADS, DUAL>;
  // four objects, not one: an LDS read then only waits for the loads into its own
  __shared__ __attribute__((aligned(1024))) unsigned char a0[SA::BYTES], a1[SA::BYTES], b0[SB::BYTES], b1[SB::BYTES];
  if (a.skip && *a.skip) return;
  const MmTile w = mm_tile(a);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), wm = wave / WGN, wn = wave % WGN;
  const int64_t m0 = (int64_t)w.m * BM, n0 = (int64_t)w.n * BN;
  const int last = (int)((a.row_bytes + 127) / 128);
  SA from_a;
  SB from_b;
  from_a.init(a.a, w.of, m0, a.row_bytes, t);
  from_b.init(a.b, w.of, DUAL ? n0 / 2 : n0, a.row_bytes, t);
  auto fetch = [&](auto* la, auto* lb, int kt) {  // behind the last tile: zeros, so that there is no branch among the products
    from_a.load(la, (int64_t)kt * 128, wave, kt < last);
    from_b.load(lb, (int64_t)kt * 128, wave, kt < last);
  };
  unsigned at_a[4], at_b[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const unsigned c = ((s * 2 + (lane >> 5)) ^ ((lane >> 1) & 7)) * 16;
    at_a[s] = (wm * TM * 32 + (lane & 31)) * 128 + c;
    at_b[s] = (wn * TN * 32 + (lane & 31)) * 128 + c;
  }
  Sum acc[TM][TN];
#pragma unroll
  for (int x = 0; x < TM; ++x)
#pragma unroll
    for (int y = 0; y < TN; ++y) acc[x][y] = Sum{};
  struct Step {
    Reg a[TM], b[TN];
  };
  auto read = [&](auto* la, auto* lb, int s, Step& to) {
#pragma unroll
    for (int x = 0; x < TM; ++x) to.a[x] = *reinterpret_cast<const JZ_LDS Reg*>((const JZ_LDS unsigned char*)la + at_a[s] + x * 4096);
#pragma unroll
    for (int y = 0; y < TN; ++y) to.b[y] = *reinterpret_cast<const JZ_LDS Reg*>((const JZ_LDS unsigned char*)lb + at_b[s] + y * 4096);
  };
  auto multiply = [&](const Step& p, const Step& q) {
#pragma unroll
    for (int x = 0; x < TM; ++x)
#pragma unroll
      for (int y = 0; y < TN; ++y) acc[x][y] = E::mfma(q.b[y], p.a[x], acc[x][y]);
  };
  constexpr int MULT = TM * TN, LOADS = SA::EACH + SB::EACH;
  // The products of a tile's last step run while its successor's first operands are read and the tile behind that is asked for.
  Step p = {}, q = {}, r = {};  // the first tile has no predecessor: zeros
  auto tile = [&](auto* la, auto* lb, auto* na, auto* nb, int kt) {
    all_landed();
    read(la, lb, 0, p);
    fetch(na, nb, kt + 1);
    if constexpr (E::SPLIT) {
      // q, r: the second half's hi and lo
      multiply(r, q);
      multiply(q, r);
      spread_out<2 * MULT, READS, LOADS>();
      read(la, lb, 2, r);
      multiply(p, p);
      spread_out<MULT, READS, 0>();
      read(la, lb, 1, q);
      multiply(r, p);
      multiply(p, r);
      spread_out<2 * MULT, READS, 0>();
      read(la, lb, 3, r);
      multiply(q, q);
      spread_out<MULT, READS, 0>();
    } else {
      multiply(q, q);
      spread_out<MULT, READS, LOADS>();
      read(la, lb, 1, q);
      multiply(p, p);
      spread_out<MULT, READS, 0>();
      read(la, lb, 2, p);
      multiply(q, q);
      spread_out<MULT, READS, 0>();
      read(la, lb, 3, q);
      multiply(p, p);
      spread_out<MULT, READS, 0>();
    }
  };
  fetch(a0, b0, 0);
  for (int kt = 0; kt < last; kt += 2) {
    tile(a0, b0, a1, b1, kt);
    if (kt + 1 < last) tile(a1, b1, a0, b0, kt + 1);
  }
  if constexpr (E::SPLIT) {
    multiply(r, q);
    multiply(q, r);
  } else {
    multiply(q, q);
  }
  all_landed();  // zeros too: the results take the operands' place
  constexpr int WIDE = TN % 2 ? 1 : TN, STRIP = 32 * WIDE * 128, FIT = SA::BYTES / STRIP;
  static_assert(FIT >= 1 && 2 * FIT >= WGM * WGN, "the results pass through the place of A");
  const MmStrip<E, WIDE> strip = {(JZ_LDS unsigned char*)(wave < FIT ? a0 + wave * STRIP : a1 + (wave - FIT) * STRIP)};
  static_for<0, TM * TN / WIDE>([&](auto I) {
    constexpr int x = decltype(I)::value / (TN / WIDE), y = decltype(I)::value % (TN / WIDE) * WIDE;
    strip.put(&acc[x][y], lane);
    epi.strip(strip, w, m0 + (wm * TM + x) * 32, n0 + (wn * TN + y) * 32, lane);
  });
}

// Few tiles: 64 x 64 by four wavefronts of 32 x 32.  What such a launch waits for is the way from memory, so four tiles of operands are on it at a time, in registers; two are in LDS.
// (X X^T of 128 x 512, ElemSplit: 10.6 us with two stages of LDS-direct loads, which wait for each other, 8.5 so.)
template <class E, class Epi>
__global__ __launch_bounds__(256, 2) void mm_small(MmArgs a, Epi epi) {
  constexpr int DEPTH = 4, EACH = 2;
  typedef typename E::Reg Reg;
  typedef typename E::Sum Sum;
  typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2][16384];
  if (a.skip && *a.skip) return;
  const MmTile w = mm_tile(a);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, wm = wave >> 1, wn = wave & 1;
  const int64_t m0 = (int64_t)w.m * 64, n0 = (int64_t)w.n * 64;
  const int last = (int)((a.row_bytes + 127) / 128);
  MmSource<64, 256, false> from_a, from_b;
  from_a.init(a.a, w.of, m0, a.row_bytes, t);
  from_b.init(a.b, w.of, n0, a.row_bytes, t);
  u32x4 ra[DEPTH][EACH], rb[DEPTH][EACH];
  auto fetch = [&](int d, int kt) {  // behind the last tile: zeros
    from_a.get(ra[d], (int64_t)kt * 128, kt < last);
    from_b.get(rb[d], (int64_t)kt * 128, kt < last);
  };
  unsigned at_a[4], at_b[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    const unsigned c = ((s * 2 + (lane >> 5)) ^ ((lane >> 1) & 7)) * 16;
    at_a[s] = (wm * 32 + (lane & 31)) * 128 + c;
    at_b[s] = 8192 + (wn * 32 + (lane & 31)) * 128 + c;
  }
  Sum acc[1] = {Sum{}};
  static_for<0, DEPTH>([&](auto D) { fetch(decltype(D)::value, decltype(D)::value); });
  for (int kt = 0; kt < last; kt += DEPTH) {
    static_for<0, DEPTH>([&](auto D) {
      constexpr int d = decltype(D)::value;
      JZ_LDS unsigned char* const to = (JZ_LDS unsigned char*)lds[d & 1];
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        *reinterpret_cast<JZ_LDS u32x4*>(to + (i * 256 + t) * 16) = ra[d][i];
        *reinterpret_cast<JZ_LDS u32x4*>(to + 8192 + (i * 256 + t) * 16) = rb[d][i];
      }
      fetch(d, kt + d + DEPTH);
      // the other place's reads were waited for before the last barrier
      lds_meet();
      Reg x[4], y[4];
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        x[s] = *reinterpret_cast<const JZ_LDS Reg*>(to + at_a[s]);
        y[s] = *reinterpret_cast<const JZ_LDS Reg*>(to + at_b[s]);
      }
      if constexpr (E::SPLIT) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          acc[0] = E::mfma(y[s], x[s], acc[0]);
          acc[0] = E::mfma(y[s], x[s + 2], acc[0]);
          acc[0] = E::mfma(y[s + 2], x[s], acc[0]);
        }
      } else {
#pragma unroll
        for (int s = 0; s < 4; ++s) acc[0] = E::mfma(y[s], x[s], acc[0]);
      }
    });
  }
  __syncthreads();  // the results take the operands' place
  const MmStrip<E, 1> strip = {(JZ_LDS unsigned char*)lds[0] + wave * 4096};
  strip.put(acc, lane);
  epi.strip(strip, w, m0 + wm * 32, n0 + wn * 32, lane);
}

// Fewer still, and short sums: 32 x 32 by eight wavefronts that share k, 64 bytes of it at a time each, straight into the registers that the matrix instructions take; four such pieces are on
// their way at a time, and nobody waits for another but for the sums, which meet in LDS and are added in the wavefronts' order.  X X^T of 128 x 512 7.4 us, 352 x 352 x 352 7 (mm_small 8.4).
// Four of them are what any launch takes here that reads what the launch before it wrote.
template <class E, class Epi>
__global__ __launch_bounds__(512, 2) void mm_tiny(MmArgs a, Epi epi) {
  constexpr int WAVES = 8, U = 4;
  typedef typename E::Reg Reg;
  typedef typename E::Sum Sum;
  typedef MmStrip<E, 1> Strip;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[WAVES][4096];
  if (a.skip && *a.skip) return;
  const MmTile w = mm_tile(a);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t m0 = (int64_t)w.m * 32, n0 = (int64_t)w.n * 32;
  const unsigned matrix = w.of / a.splits, part = w.of - matrix * a.splits;
  auto source = [&](const MmOperand& o, int64_t row0) {
    const int64_t span = (o.rows - row0 - 1) * o.pitch + a.row_bytes;
    return __builtin_amdgcn_make_buffer_rsrc((void*)(static_cast<const char*>(o.p[0]) + matrix * o.of + row0 * o.pitch), 0, (int)(span < 0x7ffffff0 ? span : 0x7ffffff0), 0x00020000);
  };
  const auto from_a = source(a.a, m0), from_b = source(a.b, n0);
  const unsigned row_a = (unsigned)((lane & 31) * a.a.pitch), row_b = (unsigned)((lane & 31) * a.b.pitch);
  const int all = (int)((a.row_bytes + 63) / 64), first = (int)((int64_t)all * part / a.splits), units = (int)((int64_t)all * (part + 1) / a.splits);
  struct Piece {
    Reg a[2], b[2];
  };
  auto get = [&](Piece& p, int u) {  // behind the end: zeros
    // ElemSplit: 16 k of high parts and, 64 bytes on, their low parts; the others: 64 bytes of k
    const unsigned j = u & 1, k0 = (unsigned)(u >> 1) * 128, h = lane >> 5, behind = u >= units ? 0x80000000u : 0u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned k = k0 + (E::SPLIT ? (2 * j + h) * 16 + i * 64 : (4 * j + 2 * i + h) * 16);
      const unsigned end = k >= (unsigned)a.row_bytes ? 0x80000000u : behind;
      p.a[i] = __builtin_bit_cast(Reg, __builtin_amdgcn_raw_buffer_load_b128(from_a, (int)((row_a + k) | end), 0, 0));
      p.b[i] = __builtin_bit_cast(Reg, __builtin_amdgcn_raw_buffer_load_b128(from_b, (int)((row_b + k) | end), 0, 0));
    }
  };
  Sum acc[1] = {Sum{}};
  auto multiply = [&](const Piece& p) {
    if constexpr (E::SPLIT) {
      acc[0] = E::mfma(p.b[0], p.a[0], acc[0]);
      acc[0] = E::mfma(p.b[0], p.a[1], acc[0]);
      acc[0] = E::mfma(p.b[1], p.a[0], acc[0]);
    } else {
      acc[0] = E::mfma(p.b[0], p.a[0], acc[0]);
      acc[0] = E::mfma(p.b[1], p.a[1], acc[0]);
    }
  };
  Piece p[2][U];
  auto ask = [&](Piece (&to)[U], int u0) {
#pragma unroll
    for (int u = 0; u < U; ++u) get(to[u], u0 + u * WAVES);
  };
  ask(p[0], first + wave);
  for (int u0 = first + wave; u0 < units; u0 += 2 * U * WAVES) {
    ask(p[1], u0 + U * WAVES);
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(p[0][u]);
    if (u0 + U * WAVES >= units) break;
    ask(p[0], u0 + 2 * U * WAVES);
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(p[1][u]);
  }
  Strip{(JZ_LDS unsigned char*)lds[wave]}.put(acc, lane);
  __syncthreads();
  if (t < 256) {
    typedef typename Strip::V4 V4;
    JZ_LDS V4* const mine = reinterpret_cast<JZ_LDS V4*>((JZ_LDS unsigned char*)lds[0] + t * 16);
    V4 v = *mine;
#pragma unroll
    for (int q = 1; q < WAVES; ++q) v += mine[q * 256];
    *mine = v;
  }
  __syncthreads();
  if (wave == 0) epi.strip(Strip{(JZ_LDS unsigned char*)lds[0]}, w, m0, n0, lane);
}

// The tile with the least expected time, in microseconds: a launch's own, what comes before and after the sums that a compute unit forms one after the other (`slots` workgroups at a time), and for
// each 128 bytes of a sum how many turns there are and what all workgroups take of the chip, whose clock falls with the matrix instructions; few workgroups wait for memory alone.
struct MmTime {
  int64_t tile;
  double launch, turn, least, each, all;
  int slots;
  double better;  // taken where it is that much of the time of the ones before
};
template <int N>
int64_t mm_tile_for(const MmTime (&kinds)[N], int64_t rows_m, int64_t rows_n, bool symmetric, int64_t count, int64_t row_bytes) {
  int64_t best = 0;
  double least = INFINITY;
  for (const MmTime& k : kinds) {
    const int64_t m = (rows_m + k.tile - 1) / k.tile, n = (rows_n + k.tile - 1) / k.tile, tiles = (symmetric ? m * (m + 1) / 2 : m * n) * count;
    const double turns = (double)((tiles + k.slots - 1) / k.slots);
    const double t = k.launch + k.turn * turns + (double)((row_bytes + 127) / 128) * std::max(k.least, turns * k.each + (double)tiles * k.all);
    if (best == 0 || t < least * k.better) {
      least = t;
      best = k.tile;
    }
  }
  return best;
}

constexpr int64_t MM_LANES = int64_t(1) << 32;  // a launch has fewer

// A launch over `count` matrices, TILE x TILE: 256 by eight wavefronts in 2 x 4, 192 and 128 by four in 2 x 2, 64: mm_small, 32: mm_tiny.
template <class E, class Epi, int TILE, bool DUAL>
int mm_launch(MmArgs a, const Epi& epi, int64_t rows_m, int64_t rows_n, int64_t count, hipStream_t st) {
  static_assert(!DUAL || TILE != 192, "");
  constexpr int WGM = 2, WGN = TILE == 256 ? 4 : 2, THREADS = TILE == 32 ? 512 : 64 * WGM * WGN;
  a.tiles_m = (int)((rows_m + TILE - 1) / TILE);
  a.tiles_n = (int)((rows_n + TILE - 1) / TILE);
  a.tiles = a.symmetric ? (unsigned)a.tiles_m * (a.tiles_m + 1) / 2 : (unsigned)a.tiles_m * a.tiles_n;
  a.workgroups = (unsigned)(a.tiles * count) * (a.splits > 1 ? a.splits : 1);
  if (a.splits < 1) a.splits = 1;
  constexpr unsigned most = (unsigned)(MM_LANES / THREADS - 1);
  for (a.first = 0; a.first < a.workgroups; a.first += most) {
    const unsigned grid = std::min(a.workgroups - a.first, most);
    if constexpr (TILE == 32) mm_tiny<E, Epi><<<grid, 512, 0, st>>>(a, epi);
    else if constexpr (TILE == 64) mm_small<E, Epi><<<grid, 256, 0, st>>>(a, epi);
    else mm_tiles<E, Epi, TILE, TILE, WGM, WGN, DUAL><<<grid, THREADS, 0, st>>>(a, epi);
  }
  return jz::launch_status();
}
