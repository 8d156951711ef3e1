// The kernels of jz_norm.hip as they stand, compiled for the host and run lane by lane, for what no timing on a GPU decides: wavefronts of a workgroup may be
// any distance apart between two barriers.  Here they run one after the other, in rising or in falling order, each as far as the next barrier.  A wavefront's lanes run
// in lock step on the GPU; here the lane whose vector reaches into a neighbour's elements runs first, so that it has loaded before the neighbour stores, as there.
// KERNELS is a file with the kernels' text.  Prints one line for every element that is not the formula's and ends with their number (0 to 100).
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <vector>

struct Dim {
  unsigned x, y;
};
enum { RUN, WAVE, GROUP, DONE };
struct Lane_ {
  ucontext_t at;
  int state;
};
static std::vector<Lane_> lanes;
static std::vector<char> stacks;
static ucontext_t scheduler;
static unsigned now_running;
static float swap_place[1024];
static Dim blockIdx, gridDim;

static void yield_(int state) {
  const unsigned me = now_running;
  lanes[me].state = state;
  swapcontext(&lanes[me].at, &scheduler);
}
static Dim lane_index() { return Dim{now_running, 0}; }
static float shuffle_xor(float v, int d) {
  const unsigned me = now_running;
  swap_place[me] = v;
  yield_(WAVE);
  const float r = swap_place[me ^ (unsigned)d];
  yield_(WAVE);
  return r;
}
static void meet() { yield_(GROUP); }

#define threadIdx lane_index()
#define __device__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __shfl_xor shuffle_xor
#define __syncthreads meet
#define __builtin_amdgcn_fence(...)
#define __builtin_amdgcn_s_barrier meet

#include "jz_vec.h"
#include KERNELS

static void (*kernel)(NormArgs);
static NormArgs args;
static void lane_main() {
  kernel(args);
  lanes[now_running].state = DONE;
}
// one workgroup; `first`: the lane of its wavefront that goes first
static void run_group(unsigned threads, bool falling, int first) {
  constexpr size_t STACK = 64 << 10;
  lanes.resize(threads);
  stacks.resize(STACK * threads);
  for (unsigned t = 0; t < threads; ++t) {
    getcontext(&lanes[t].at);
    lanes[t].at.uc_stack.ss_sp = &stacks[STACK * t];
    lanes[t].at.uc_stack.ss_size = STACK;
    lanes[t].at.uc_link = &scheduler;
    lanes[t].state = RUN;
    makecontext(&lanes[t].at, lane_main, 0);
  }
  const unsigned waves = threads / 64;
  for (;;) {
    bool done = true;
    for (unsigned q = 0; q < waves; ++q) {
      const unsigned w = falling ? waves - 1 - q : q;
      for (bool going = true; going;) {
        going = false;
        for (unsigned i = 0; i < 64; ++i) {
          const unsigned t = w * 64 + ((unsigned)first % 64 + i) % 64;
          if (lanes[t].state == GROUP || lanes[t].state == DONE) continue;
          now_running = t;
          swapcontext(&scheduler, &lanes[t].at);
          going = going || lanes[t].state == WAVE;
        }
      }
    }
    for (Lane_& l : lanes) {
      if (l.state == GROUP) l.state = RUN;
      done = done && l.state == DONE;
    }
    if (done) return;
  }
}

static int wrong = 0;
static void compare(const char* what, int C, bool falling, const std::vector<float>& got, const std::vector<double>& want) {
  for (size_t i = 0; i < want.size(); ++i)
    if (!(fabs(got[i] - want[i]) <= 1e-4 * (1 + fabs(want[i])))) {
      if (wrong < 100) printf("%s, %d channels, wavefronts %s: row %zu, channel %zu: %g, exact %g\n", what, C, falling ? "falling" : "rising", i / C, i % C, got[i], want[i]), ++wrong;
      break;
    }
}
static float value(unsigned i) { return (float)((i * 2654435761u >> 8) & 0xffff) / 32768.f - 1.f + 1e-3f; }

template <int MODE, int FT, int FNV, int BT, int BNV>
static void width(int C, bool post, bool backward) {
  const int rows = 2;
  const size_t e = (size_t)rows * C;
  std::vector<float> r(e), y(e), gate(C), w_post(C), w_pre(C), dn(e), dr_out(e);
  for (size_t i = 0; i < e; ++i) r[i] = value(i), y[i] = value(i + 77777), dn[i] = value(i + 333), dr_out[i] = value(i + 4444);
  for (int i = 0; i < C; ++i) gate[i] = value(i + 5), w_post[i] = 1 + value(i + 9) / 4, w_pre[i] = 1 + value(i + 3) / 4;
  const double eps = 1e-5, a = 0.75, s = 1.5;
  std::vector<double> want_r(e), want_n(e), want_dr(e), want_dy(e);
  std::vector<float> k1(rows), k2(rows);
  for (int m = 0; m < rows; ++m) {
    double q1 = 0, q2 = 0, c1 = 0, c2 = 0;
    const size_t o = (size_t)m * C;
    for (int i = 0; i < C; ++i) q1 += (double)y[o + i] * y[o + i];
    const double d1 = post ? 1 / sqrt(q1 / C + eps) : 1;
    for (int i = 0; i < C; ++i) {
      want_r[o + i] = a * r[o + i] + s * gate[i] * y[o + i] * d1 * (post ? w_post[i] : 1.);
      q2 += want_r[o + i] * want_r[o + i];
    }
    const double d2 = 1 / sqrt(q2 / C + eps);
    for (int i = 0; i < C; ++i) want_n[o + i] = want_r[o + i] * d2 * w_pre[i], c2 += dn[o + i] * w_pre[i] * want_r[o + i] * d2 / C;
    std::vector<double> dp(C);
    for (int i = 0; i < C; ++i) {
      const double R = dr_out[o + i] + d2 * (w_pre[i] * dn[o + i] - want_r[o + i] * d2 * c2);
      want_dr[o + i] = a * R;
      dp[i] = s * gate[i] * R;
      if (post) c1 += w_post[i] * dp[i] * y[o + i] * d1 / C;
    }
    for (int i = 0; i < C; ++i) want_dy[o + i] = post ? d1 * (w_post[i] * dp[i] - y[o + i] * d1 * c1) : dp[i];
    k1[m] = (float)d1;
    k2[m] = (float)d2;
  }
  // the last vector's lane goes first in its wavefront
  const int first = (C - 1) / 8 % (backward ? BT : FT);
  for (bool falling : {false, true}) {
    std::vector<float> stream = backward ? dr_out : r, n(e), out_y(e), r1(rows), r2(rows), dw(C), dg(C), dq(C), part(4 * C), kept(want_r.begin(), want_r.end());
    args = NormArgs{};
    args.rows = args.rows_per_group = rows;
    args.C = C;
    args.eps = (float)eps;
    args.res_scale = (float)a;
    args.branch_scale = (float)s;
    args.inv_c = 1.f / C;
    args.y = y.data();
    args.w_post = post ? w_post.data() : nullptr;
    args.gate = gate.data();
    args.w_pre = w_pre.data();
    if (!backward) {
      args.r = args.r_out = stream.data();
      args.n = n.data();
      args.rstd_post = r1.data();
      args.rstd_pre = r2.data();
      constexpr int ROWS = FT >= 256 ? 1 : 256 / FT;
      kernel = norm_fwd<float, float, MODE, FT, FNV>;
      gridDim = Dim{(unsigned)((rows + ROWS - 1) / ROWS), 1};
      for (blockIdx.x = 0; blockIdx.x < gridDim.x; ++blockIdx.x) run_group(FT >= 256 ? FT : 256, falling, first);
      compare(post ? "r_out with a post-norm" : "r_out", C, falling, stream, want_r);
      compare(post ? "n with a post-norm" : "n", C, falling, n, want_n);
    } else {
      args.r_out = kept.data();
      args.rstd_post = k1.data();
      args.rstd_pre = k2.data();
      args.dr_out = args.dr = stream.data();
      args.dn = dn.data();
      args.dy = out_y.data();
      args.dw_post = post ? dw.data() : nullptr;
      args.dgate = dg.data();
      args.dw_pre = dq.data();
      args.part = part.data();
      args.slab = rows;
      args.slabs = 1;
      args.step = 1;
      kernel = norm_bwd<float, float, MODE, BT, BNV, BT < 1024 ? BLOCK : ANY>;
      gridDim = Dim{1, 1};
      blockIdx.x = 0;
      run_group(BT, falling, first);
      compare(post ? "dr with a post-norm" : "dr", C, falling, stream, want_dr);
      compare(post ? "dy with a post-norm" : "dy", C, falling, out_y, want_dy);
    }
  }
}
// the lanes that a width's launch takes (with_lanes, behind the kernels in jz_norm.hip)
static void width(int C, bool post, bool backward) {
  if (C % 8 == 0) return;
  if (C <= 512) width<RAGGED, 64, 1, 64, 1>(C, post, backward);
  else if (C <= 1024) width<RAGGED, 64, 2, 128, 1>(C, post, backward);
  else if (C <= 2048) width<RAGGED, 256, 1, 256, 1>(C, post, backward);
  else if (C <= 4096) width<RAGGED, 256, 2, 512, 1>(C, post, backward);
  else if (C <= 8192) width<RAGGED, 512, 2, 1024, 1>(C, post, backward);
  else width<RAGGED, 1024, 2, 1024, 2>(C, post, backward);
}
int main(int argc, char** argv) {
  const bool backward = argc > 1 && atoi(argv[1]);
  for (int post = 0; post < 2; ++post) {
    // every width whose last vector begins among another wavefront's elements, and others of every kind
    for (int C = 513; C < 16384; C += 512)
      for (int i = 0; i < 7; i += backward ? 3 : 1) width(C + i, post, backward);
    for (int C : {9, 15, 100, 511, 1001, 1021, 1033, 2047, 3001, 4095, 4099, 6001, 8191, 10001, 16383}) width(C, post, backward);
  }
  printf("%d\n", wrong);
  return wrong;
}
