// Gated feed-forward block, forward and backward (include/jz.h: jz_ffn_fwd, jz_ffn_bwd): planning and entry points; the products are
// in jz_ffn_gemm.h.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "jz_internal.h"

namespace {

#include "jz_lds_dma.h"
#include "jz_vec.h"
#include "jz_ffn_gemm.h"
#include "jz_ffn_few.h"

struct FfnTensor {
  const void* p;
  size_t bytes;
  bool out;
};
int ffn_look_over(const FfnTensor* t, int n, const void* ws, size_t ws_bytes) {
  for (int i = 0; i < n; ++i)
    if (t[i].p && !jz::aligned16(t[i].p)) return JZ_ERR_ALIGN;
  for (int i = 0; i < n; ++i) {
    if (jz::overlaps(t[i].p, t[i].bytes, ws, ws_bytes)) return JZ_ERR_ALIAS;
    for (int j = i + 1; j < n; ++j)
      if ((t[i].out || t[j].out) && jz::overlaps(t[i].p, t[i].bytes, t[j].p, t[j].bytes)) return JZ_ERR_ALIAS;
  }
  return JZ_OK;
}

struct FfnShape {
  int64_t M, D, F, O, ldx, ldy, lddx, lddy;
};
int ffn_shape(const jz_ffn_desc* d, FfnShape* s) {
  if (!d) return JZ_ERR_NULL;
  if (d->rows < 0 || d->in_features <= 0 || d->hidden <= 0 || d->out_features <= 0 || d->act < JZ_ACT_SILU || d->act > JZ_ACT_RELU || d->dtype < JZ_F16 ||
      d->dtype > JZ_F32)
    return JZ_ERR_SHAPE;
  const int64_t in = d->in_features, out = d->out_features;
  *s = {d->rows, in, d->hidden, out, d->x_stride ? d->x_stride : in, d->y_stride ? d->y_stride : out, d->dx_stride ? d->dx_stride : in,
        d->dy_stride ? d->dy_stride : out};
  if (s->ldx < in || s->ldy < out || s->lddx < in || s->lddy < out) return JZ_ERR_SHAPE;
  const int64_t most = int64_t(1) << 24, wide = std::max(std::max(s->ldx, s->ldy), std::max(s->lddx, s->lddy));
  if (d->dtype == JZ_F32 || d->rows > (int64_t(1) << 31) || in > most || d->hidden > most || out > most || wide > most) return JZ_ERR_UNSUPPORTED;
  // tensors larger than any card's memory; below, tiles are counted in 32 bits (at most 2^27 in a launch)
  if (std::max(std::max(d->rows * std::max<int64_t>(wide, d->hidden), d->hidden * in), d->hidden * out) > int64_t(1) << 38) return JZ_ERR_UNSUPPORTED;
  return JZ_OK;
}
// bytes from the first to the last element of rows x cols with a row pitch
size_t span(int64_t rows, int64_t cols, int64_t ld) { return rows ? ((size_t)(rows - 1) * ld + cols) * 2 : 0; }

template <int BM, int BN>
void set_tiles(GemmArgs* a, int epi) {
  for (int i = 0; i < a->products; ++i) {
    a->p[i].tiles_m = (int)((a->p[i].M + BM - 1) / BM);
    const int64_t cols = epi == EPI_GLU ? 2 * ((a->p[i].N + 31) / 32 * 32) : a->p[i].N;
    a->p[i].tiles_n = (int)((cols + BN - 1) / BN);
  }
}
int tile_count(const GemmArgs& a) {
  int n = 0;
  for (int i = 0; i < a.products; ++i) n += a.p[i].tiles_m * a.p[i].tiles_n;
  return n;
}

// LDS-direct loads move 16 bytes from multiples of 16 and reach 2^31 bytes behind a tile's first row.
template <bool KCA, bool KCB>
bool direct(const GemmArgs& a) {
  for (int i = 0; i < a.products; ++i) {
    const Product& p = a.p[i];
    if (p.lda % 8 || p.ldb % 8 || p.lda >= (1 << 22) || p.ldb >= (1 << 22) || ((KCA || KCB) && p.K % 8)) return false;
    if (!p.eights && ((!KCA && p.M % 8) || (!KCB && p.N % 8))) return false;
  }
  return true;
}

// What a launch does: a tile kernel (256 x 256 or 128 x 128), how many tiles have a workgroup of their own, and how many workgroups share the sum of each of
// the others.
struct FfnPlan {
  int tile, full, splits;
};
struct Scratch {  // room for partial sums
  void* p;
  size_t bytes;
};
int64_t k_tiles(const GemmArgs& a) { return (a.p[0].K + BK - 1) / BK * a.parts; }  // the products of a launch have one K
int64_t count_tiles(const GemmArgs& a, int epi, int tile) {
  int64_t n = 0;
  for (int i = 0; i < a.products; ++i) n += ((a.p[i].M + tile - 1) / tile) * (((epi == EPI_GLU ? (a.p[i].N + 31) / 32 * 64 : a.p[i].N) + tile - 1) / tile);
  return n;
}
size_t partial_bytes(const FfnPlan& p, int64_t tiles) { return p.splits > 1 ? (size_t)(tiles - p.full) * p.splits * p.tile * p.tile * 4 : 0; }

constexpr int64_t LANES = int64_t(1) << 32;  // a launch has fewer

template <class T, bool KCA, bool KCB, int EPI, int ACT>
void launch_tiles(GemmArgs a, int tile, hipStream_t st) {
  const bool lds_direct = direct<KCA, KCB>(a);
  const unsigned threads = lds_direct && tile == 256 ? 512 : 256, most = (unsigned)(LANES / threads - 1);
  for (a.first = 0; a.first < a.workgroups; a.first += most) {
    const unsigned grid = std::min(a.workgroups - a.first, most);
    if (!lds_direct) ffn_gemm_any<T, KCA, KCB, EPI, ACT, 128, 128><<<grid, threads, 0, st>>>(a);
    else if (tile == 256) ffn_gemm<T, KCA, KCB, EPI, ACT, 256, 256, 2, 4><<<grid, threads, 0, st>>>(a);
    else ffn_gemm<T, KCA, KCB, EPI, ACT, 128, 128, 2, 2><<<grid, threads, 0, st>>>(a);
  }
}

template <class T, bool KCA, bool KCB, int EPI>
int launch(GemmArgs a, const FfnPlan& plan, const Scratch& ws, hipStream_t st) {
  if (plan.tile == 256) set_tiles<256, 256>(&a, EPI);
  else set_tiles<128, 128>(&a, EPI);
  const int tiles = tile_count(a), full = plan.splits > 1 ? plan.full : tiles, split = tiles - full;
  if (tiles <= 0) return JZ_OK;
  a.full = full;
  a.splits = plan.splits;
  a.tiles_per_split = (int)((k_tiles(a) + plan.splits - 1) / plan.splits);
  a.partial = static_cast<float*>(ws.p);
  a.workgroups = (unsigned)(full + split * plan.splits);
  if (EPI != EPI_GLU_BWD || a.act == 0) launch_tiles<T, KCA, KCB, EPI, 0>(a, plan.tile, st);
  else if constexpr (EPI == EPI_GLU_BWD) {
    if (a.act == 1) launch_tiles<T, KCA, KCB, EPI, 1>(a, plan.tile, st);
    else if (a.act == 2) launch_tiles<T, KCA, KCB, EPI, 2>(a, plan.tile, st);
    else launch_tiles<T, KCA, KCB, EPI, 3>(a, plan.tile, st);
  }
  if (jz::launch_status() != JZ_OK) return JZ_ERR_LAUNCH;
  if (split > 0) {
    const dim3 join(plan.tile * plan.tile / (EPI == EPI_GLU ? 16 : 8) / 256, split);
    if (plan.tile == 256) ffn_join<T, EPI, 256><<<join, 256, 0, st>>>(a);
    else ffn_join<T, EPI, 128><<<join, 256, 0, st>>>(a);
  }
  return jz::launch_status();
}

// The plan with the least expected time.  Microseconds, fitted to FP16 and BF16 products of 128 to 16384 rows and 1024 to 12288 features: a k tile of a
// 256 x 256 tile takes 1.22 alone on the chip and 1.75 with all 256 compute units busy (0.62 and, two workgroups a unit, 1.08 for 128 x 128), what comes before
// and after the k tiles 10 (3); joining moves the partial sums twice and is a launch.
FfnPlan choose(const GemmArgs& a, int epi, bool lds_direct, size_t ws_bytes) {
  FfnPlan best = {128, 0, 1};  // one workgroup a tile: always among the plans below
  double least = 1e30;
  const double kt = (double)k_tiles(a);
  for (int tile : {256, 128}) {
    if (tile == 256 && !lds_direct) continue;
    const int64_t tiles = count_tiles(a, epi, tile), slots = tile == 256 ? 256 : 512;
    auto tile_time = [&](double workgroups, double k) {
      const double fill = std::min(1., workgroups / slots);
      return tile == 256 ? k * (1.22 + 0.53 * fill) + 10. : k * (0.62 + 0.46 * fill) + 3.;
    };
    for (int rounds = 0; rounds < 2; ++rounds) {  // all tiles are split, or those of the last round, which does not fill the chip
      const int64_t full = rounds ? tiles / slots * slots : 0, rest = tiles - full;
      if (rounds && full == 0) continue;
      for (int s = 1; s <= 32 && (s == 1 || s <= kt); s += s < 4 ? 1 : s < 8 ? 2 : s < 16 ? 4 : 8) {
        const FfnPlan p = {tile, (int)(s == 1 ? tiles : full), s};
        if (partial_bytes(p, tiles) > ws_bytes) continue;
        const double each = std::ceil(kt / s);
        const int64_t wg = rest * s, turns = (wg + slots - 1) / slots;
        double t = full / slots * tile_time(slots, kt) + (turns ? (turns - 1) * tile_time(slots, each) + tile_time(turns > 1 ? slots : wg, each) : 0);
        if (s > 1 && rest > 0) t += 5. + (double)partial_bytes(p, tiles) * 2. / 5e6;
        if (t < least) {
          least = t;
          best = p;
        }
      }
    }
  }
  return best;
}
// room for partial sums that a plan may use
constexpr size_t PARTIAL_LIMIT = size_t(128) << 20;
size_t wanted(const GemmArgs& a, int epi, bool lds_direct) {
  const FfnPlan p = choose(a, epi, lds_direct, PARTIAL_LIMIT);
  return partial_bytes(p, count_tiles(a, epi, p.tile));
}

template <class T, bool KCA, bool KCB, int EPI>
int gemm(GemmArgs a, const Scratch& ws, hipStream_t st) {
  return launch<T, KCA, KCB, EPI>(a, choose(a, EPI, direct<KCA, KCB>(a), std::min(ws.bytes, PARTIAL_LIMIT)), ws, st);
}

template <class T, bool GLU, int TT>
int launch_few(const GemmArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)((a.p[0].N + 15) / 16);
  if (direct<true, true>(a)) {
    // stages of a wavefront's own: as many wavefronts as LDS holds, in one workgroup a compute unit or, where there are more of them, two
    constexpr int W = GLU && TT == 4 ? 4 : 8, CH = TT == 1 && !GLU ? 2 : 1;
    if (grid <= 256 || W == 4) ffn_few<T, GLU, TT, W, CH><<<grid, 64 * W, 0, st>>>(a);
    else ffn_few<T, GLU, TT, 4, CH><<<grid, 256, 0, st>>>(a);
  } else if (grid <= 256) {  // sixteen wavefronts fit a compute unit: as many to a workgroup as keep all workgroups on the chip at once
    ffn_few_any<T, GLU, TT, 16><<<grid, 1024, 0, st>>>(a);
  } else if (grid <= 512) {
    ffn_few_any<T, GLU, TT, 8><<<grid, 512, 0, st>>>(a);
  } else {
    ffn_few_any<T, GLU, TT, 4><<<grid, 256, 0, st>>>(a);
  }
  return jz::launch_status();
}
constexpr int64_t FEW_ROWS = 64;
template <class T, bool GLU>
int few(const GemmArgs& a, hipStream_t st) {
  const int64_t M = a.p[0].M;
  return M <= 16 ? launch_few<T, GLU, 1>(a, st) : M <= 32 ? launch_few<T, GLU, 2>(a, st) : launch_few<T, GLU, 4>(a, st);
}

Product product(const void* a, int64_t lda, const void* b, int64_t ldb, void* c, int64_t ldc, int64_t M, int64_t N, int64_t K) {
  Product p = {};
  p.a[0] = p.a[1] = a;
  p.b[0] = p.b[1] = b;
  p.c = c;
  p.lda = lda;
  p.ldb = ldb;
  p.ldc = ldc;
  p.M = M;
  p.N = N;
  p.K = p.k_rows = K;
  return p;
}
GemmArgs one(const Product& p, int act) {
  GemmArgs a = {};
  a.p[0] = p;
  a.products = a.parts = 1;
  a.act = act;
  return a;
}

// ---- operands ---------------------------------------------------------------------------------------------------------------
int64_t round8(int64_t n) { return (n + 7) & ~int64_t(7); }
struct Matrix {
  const void* p;
  int64_t rows, cols, ld;
};
// The LDS-direct kernels want rows that start on 16 bytes, and as operands along k rows that are a multiple of 8 long: others are copied into the workspace first,
// where it has room, since the kernel that takes any sizes runs at half their rate.  FP16, forward and backward: 8192 rows, 2047 -> 5631 features 1968 us with copies and
// 2899 without (2048 -> 5632, which needs none: 1692); 2000 rows, 1001 -> 2801 features 242 and 353; 100 rows, 2047 -> 5631 features 167 and 391.
class Aligner {
 public:
  explicit Aligner(Scratch* room) : room_(room) {}
  static size_t bytes(const Matrix& m) { return m.ld % 8 || m.cols % 8 ? (size_t)m.rows * round8(m.cols) * 2 + 255 & ~size_t(255) : 0; }
  Matrix room(const Matrix& m) {  // where the copy will lie
    const size_t n = bytes(m);
    if (!n || m.rows == 0) return m;
    const Matrix to = {room_->p, m.rows, m.cols, round8(m.cols)};
    room_->p = static_cast<char*>(room_->p) + n;
    room_->bytes -= n;
    return to;
  }
  Matrix operator()(const Matrix& m) {
    const Matrix to = room(m);
    if (to.p == m.p) return m;
    c_.m[c_.count++] = {m.p, const_cast<void*>(to.p), m.rows, m.cols, m.ld, to.ld, blocks_};
    blocks_ += (m.rows * (to.ld / 8) + 255) / 256;
    return to;
  }
  template <class T>
  int run(hipStream_t st) {
    for (c_.first = 0; c_.first < blocks_; c_.first += LANES / 256 - 1) ffn_copy<T><<<(unsigned)std::min(blocks_ - c_.first, LANES / 256 - 1), 256, 0, st>>>(c_);
    return jz::launch_status();
  }

 private:
  Scratch* room_;
  Copies c_ = {};
  int64_t blocks_ = 0;
};
// A copied row ends in zeros, which a sum may count; another's may be followed by anything.
struct Operands {
  Matrix x, wg, wu, wd, h, dy;
  bool copied;
};
Operands operands(const FfnShape& s, const void* x, const void* wg, const void* wu, const void* wd, const void* h, const void* dy) {
  return {{x, s.M, s.D, s.ldx}, {wg, s.F, s.D, s.D}, {wu, s.F, s.D, s.D}, {wd, s.O, s.F, s.F}, {h, s.M, s.F, s.F}, {dy, s.M, s.O, s.lddy}, false};
}
size_t copies_fwd(const Operands& o) { return Aligner::bytes(o.x) + Aligner::bytes(o.wg) + Aligner::bytes(o.wu) + Aligner::bytes(o.wd) + Aligner::bytes(o.h); }
size_t copies_bwd(const Operands& o) { return copies_fwd(o) + Aligner::bytes(o.dy); }

// ---- the products of the block, in the order of the calls ---------------------------------------------------------------------
GemmArgs glu_args(const FfnShape& s, int act, const Operands& o, void* h, void* gate, void* up) {
  GemmArgs a = one(product(o.x.p, o.x.ld, o.wg.p, o.wg.ld, h, s.F, s.M, s.F, s.D), act);
  if (o.copied) a.p[0].K = round8(s.D);
  a.p[0].b[1] = o.wu.p;
  a.out0 = gate;
  a.out1 = up;
  return a;
}
GemmArgs down_args(const FfnShape& s, const Operands& o, void* y) {
  GemmArgs a = one(product(o.h.p, o.h.ld, o.wd.p, o.wd.ld, y, s.ldy, s.M, s.O, s.F), 0);
  if (o.copied) a.p[0].K = round8(s.F);
  return a;
}
GemmArgs dh_args(const FfnShape& s, int act, const Operands& o, const void* gate, const void* up, void* dgate, void* dup) {
  GemmArgs a = one(product(o.dy.p, o.dy.ld, o.wd.p, o.wd.ld, nullptr, round8(s.F), s.M, s.F, s.O), act);
  if (o.copied) a.p[0].K = round8(s.O);
  a.p[0].eights = o.copied;
  a.gate = gate;
  a.up = up;
  a.out0 = dgate;
  a.out1 = dup;
  return a;
}
GemmArgs dx_args(const FfnShape& s, const Operands& o, const void* dgate, const void* dup, void* dx) {
  GemmArgs a = one(product(dgate, round8(s.F), o.wg.p, o.wg.ld, dx, s.lddx, s.M, s.D, s.F), 0);
  a.p[0].K = round8(s.F);  // dgate and dup always end in zeros
  a.p[0].eights = o.copied;
  a.p[0].a[1] = dup;
  a.p[0].b[1] = o.wu.p;
  a.parts = 2;
  return a;
}
GemmArgs dw_args(const FfnShape& s, const Operands& o, const void* dgate, const void* dup, void* dwg, void* dwu, void* dwd) {
  GemmArgs a = one(product(dgate, round8(s.F), o.x.p, o.x.ld, dwg, s.D, s.F, s.D, s.M), 0);
  a.p[1] = product(dup, round8(s.F), o.x.p, o.x.ld, dwu, s.D, s.F, s.D, s.M);
  a.p[2] = product(o.dy.p, o.dy.ld, o.h.p, o.h.ld, dwd, s.F, s.O, s.F, s.M);
  a.products = 3;
  for (Product& p : a.p) p.eights = o.copied;
  return a;
}
// the same with every operand that would be copied as its copy will be, for planning
Operands aligned_shapes(Operands o) {
  for (Matrix* m : {&o.x, &o.wg, &o.wu, &o.wd, &o.h, &o.dy})
    if (Aligner::bytes(*m)) m->ld = round8(m->cols);
  o.copied = true;
  return o;
}

template <class T>
int run_fwd(const FfnShape& s, int act, Operands o, void* h, void* gate, void* up, void* y, Scratch ws, hipStream_t st) {
  if (s.M <= FEW_ROWS) {
    const int rc = few<T, true>(glu_args(s, act, o, h, gate, up), st);
    return rc == JZ_OK ? few<T, false>(down_args(s, o, y), st) : rc;
  }
  o.copied = copies_fwd(o) <= ws.bytes;
  if (o.copied) {
    Aligner align(&ws);
    o.x = align(o.x);
    o.wg = align(o.wg);
    o.wu = align(o.wu);
    o.wd = align(o.wd);
    o.h = align.room(o.h);
    const int rc = align.run<T>(st);
    if (rc != JZ_OK) return rc;
  }
  GemmArgs first = glu_args(s, act, o, h, gate, up);
  if (o.h.p != h) {  // the first product writes both
    first.padded = const_cast<void*>(o.h.p);
    first.ld_padded = o.h.ld;
  }
  const int rc = gemm<T, true, true, EPI_GLU>(first, ws, st);
  return rc == JZ_OK ? gemm<T, true, true, EPI_STORE>(down_args(s, o, y), ws, st) : rc;
}

template <class T>
int run_bwd(const FfnShape& s, int act, Operands o, const void* gate, const void* up, void* dx, void* dwg, void* dwu, void* dwd, void* dgate, void* dup, Scratch ws,
            hipStream_t st) {
  o.copied = copies_bwd(o) <= ws.bytes;
  if (o.copied) {
    Aligner align(&ws);
    if (dwg) {
      o.x = align(o.x);
      o.h = align(o.h);
    }
    if (dx) {
      o.wg = align(o.wg);
      o.wu = align(o.wu);
    }
    o.wd = align(o.wd);
    o.dy = align(o.dy);
    const int rc = align.run<T>(st);
    if (rc != JZ_OK) return rc;
  }
  int rc = gemm<T, true, false, EPI_GLU_BWD>(dh_args(s, act, o, gate, up, dgate, dup), ws, st);
  if (rc == JZ_OK && dx) rc = gemm<T, true, false, EPI_STORE>(dx_args(s, o, dgate, dup, dx), ws, st);
  if (rc == JZ_OK && dwg) rc = gemm<T, false, false, EPI_STORE>(dw_args(s, o, dgate, dup, dwg, dwu, dwd), ws, st);
  return rc;
}

size_t hidden_bytes(const FfnShape& s) { return ((size_t)s.M * round8(s.F) * 2 + 255) & ~size_t(255); }

}  // namespace

extern "C" int jz_ffn_fwd_workspace_bytes(const jz_ffn_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  FfnShape s;
  const int rc = ffn_shape(d, &s);
  if (rc != JZ_OK) return rc;
  const Operands o = operands(s, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr), al = aligned_shapes(o);
  const GemmArgs a = glu_args(s, 0, al, nullptr, nullptr, nullptr), b = down_args(s, al, nullptr);
  *bytes = s.M <= FEW_ROWS ? 0 : copies_fwd(o) + std::max(wanted(a, EPI_GLU, direct<true, true>(a)), wanted(b, EPI_STORE, direct<true, true>(b)));
  return JZ_OK;
}

extern "C" int jz_ffn_bwd_workspace_bytes(const jz_ffn_desc* d, size_t* bytes) {
  if (!bytes) return JZ_ERR_NULL;
  FfnShape s;
  const int rc = ffn_shape(d, &s);
  if (rc != JZ_OK) return rc;
  const Operands o = operands(s, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr), al = aligned_shapes(o);
  const GemmArgs a = dh_args(s, 0, al, nullptr, nullptr, nullptr, nullptr), b = dx_args(s, al, nullptr, nullptr, nullptr),
                 c = dw_args(s, al, nullptr, nullptr, nullptr, nullptr, nullptr);
  *bytes = 2 * hidden_bytes(s) + copies_bwd(o) + std::max(wanted(a, EPI_GLU_BWD, direct<true, false>(a)),
                                                          std::max(wanted(b, EPI_STORE, direct<true, false>(b)), wanted(c, EPI_STORE, direct<false, false>(c))));
  return JZ_OK;
}

extern "C" int jz_ffn_fwd(const jz_ffn_desc* d, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* h, void* gate, void* up, void* y,
                          void* ws, size_t ws_bytes, void* hip_stream) {
  FfnShape s;
  int rc = ffn_shape(d, &s);
  if (rc != JZ_OK) return rc;
  if (!w_gate || !w_up || !w_down || (s.M && (!x || !h || !y || !gate != !up))) return JZ_ERR_NULL;
  if (s.M == 0) return JZ_OK;
  const size_t hid = span(s.M, s.F, s.F), w = span(s.F, s.D, s.D);
  const FfnTensor t[] = {{x, span(s.M, s.D, s.ldx), false}, {w_gate, w, false}, {w_up, w, false}, {w_down, span(s.O, s.F, s.F), false}, {h, hid, true},
                         {gate, hid, true}, {up, hid, true}, {y, span(s.M, s.O, s.ldy), true}};
  if (ws_bytes && !ws) return JZ_ERR_WORKSPACE;
  if (ws && !jz::aligned16(ws)) return JZ_ERR_ALIGN;
  rc = ffn_look_over(t, 8, ws, ws_bytes);
  if (rc != JZ_OK) return rc;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const Operands o = operands(s, x, w_gate, w_up, w_down, h, nullptr);
  const Scratch room = {ws, ws_bytes};
  return d->dtype == JZ_F16 ? run_fwd<_Float16>(s, d->act, o, h, gate, up, y, room, st) : run_fwd<__bf16>(s, d->act, o, h, gate, up, y, room, st);
}

extern "C" int jz_ffn_bwd(const jz_ffn_desc* d, const void* x, const void* w_gate, const void* w_up, const void* w_down, const void* gate, const void* up,
                          const void* h, const void* dy, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* ws, size_t ws_bytes, void* hip_stream) {
  FfnShape s;
  int rc = ffn_shape(d, &s);
  if (rc != JZ_OK) return rc;
  const bool weights = dw_gate || dw_up || dw_down;
  if (!w_gate || !w_up || !w_down || (weights && (!dw_gate || !dw_up || !dw_down))) return JZ_ERR_NULL;
  if (s.M && (!gate || !up || !dy || (weights && (!x || !h)) || (!dx && !weights))) return JZ_ERR_NULL;
  const size_t need = 2 * hidden_bytes(s);
  if (ws_bytes < need || (ws_bytes && !ws)) return JZ_ERR_WORKSPACE;
  if (ws && !jz::aligned16(ws)) return JZ_ERR_ALIGN;
  const size_t hid = span(s.M, s.F, s.F), w = span(s.F, s.D, s.D), w2 = span(s.O, s.F, s.F);
  const FfnTensor t[] = {{weights ? x : nullptr, span(s.M, s.D, s.ldx), false}, {w_gate, w, false}, {w_up, w, false}, {w_down, w2, false}, {gate, hid, false}, {up, hid, false},
                         {weights ? h : nullptr, hid, false}, {dy, span(s.M, s.O, s.lddy), false}, {dx, span(s.M, s.D, s.lddx), true}, {dw_gate, w, true}, {dw_up, w, true},
                         {dw_down, w2, true}};
  rc = ffn_look_over(t, 12, ws, ws_bytes);
  if (rc != JZ_OK) return rc;
  char* b = static_cast<char*>(ws);
  void *dgate = b, *dup = b + hidden_bytes(s);
  const Scratch rest{b + need, ws_bytes - need};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const Operands o = operands(s, x, w_gate, w_up, w_down, h, dy);
  return d->dtype == JZ_F16 ? run_bwd<_Float16>(s, d->act, o, gate, up, dx, dw_gate, dw_up, dw_down, dgate, dup, rest, st)
                            : run_bwd<__bf16>(s, d->act, o, gate, up, dx, dw_gate, dw_up, dw_down, dgate, dup, rest, st);
}
