"""jz_norm_residual_fwd and jz_norm_residual_bwd against their formulas in 64 bits.

Tolerances, in FP32 roundings (2^-24) of the size of the terms that a result is added up from.  A row's sum of squares is at most 16 squares a
lane, summed in pairs, and a tree over lanes and wavefronts: 16 + 3 + 6 + 16 additions at most, all of one sign; the root halves it: rstd is within
25 roundings, and a product of it with the rest within 32.  n has that twice (through r_out and its own rstd): 64.  Backward a row mean of products
takes the same sum, without the root, of terms within 8 roundings: 64, and through the gradient of the second norm twice: 128.  The sums over rows take
at most 32 rows in a lane and a quarter of 512 slabs one after the other: 176 additions on top of their terms' 128, 320 in all.  The backward call is
compared on the tensors it is given, the forward call's rounded ones."""
import numpy as np
import pytest
import torch

from oracle import blocks
from jzt_blocks import DEV, TYPES, check, nans, randn, wide

pytestmark = pytest.mark.gpu
EPS, RES, BRANCH = 1e-5, 0.75, 1.5


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


class Case:
    def __init__(self, jz, rows, C, dtype="f16", res=None, per=0, post=True, gate=True, pre=True, branch=True, seed=0):
        g = np.random.default_rng((rows, C, per, seed))
        t, rt = TYPES[dtype], TYPES[res or dtype]
        self.jz, self.rows, self.C, self.t, self.rt, self.branch, self.pre = jz, rows, C, t, rt, branch, pre
        self.groups = rows // per if per else 1
        self.desc = jz.norm_residual_desc(rows, C, per, jz.dtype_of(t), jz.dtype_of(rt), EPS, RES, BRANCH)
        f = torch.float32
        self.r, self.y = randn(g, (rows, C), rt, 2.0), randn(g, (rows, C), t, 0.7) if branch else None
        self.w_post = randn(g, (C,), f, 0.3, 1.0) if post and branch else None
        self.gate = randn(g, (self.groups, C), f) if gate and branch else None
        self.w_pre = randn(g, (C,), f, 0.3, 1.0) if pre else None
        self.dr_out, self.dn = randn(g, (rows, C), rt), randn(g, (rows, C), t) if pre else None

    def forward(self):
        self.r_out = nans((self.rows, self.C), self.rt) if self.branch else None
        self.n = nans((self.rows, self.C), self.t) if self.pre else None
        self.k1 = nans(self.rows, torch.float32) if self.w_post is not None else None
        self.k2 = nans(self.rows, torch.float32) if self.pre else None
        self.jz.jz_norm_residual_fwd(self.desc, self.r, self.y, self.w_post, self.gate, self.w_pre, self.r_out, self.n, self.k1, self.k2)
        torch.cuda.synchronize()

    def backward(self, dr_out="given"):
        e = (self.rows, self.C)
        self.dr, self.dy = nans(e, self.rt), nans(e, self.t) if self.branch else None
        self.dw_post = nans(self.C, self.t) if self.w_post is not None else None
        self.dgate = nans((self.groups, self.C), self.t) if self.gate is not None else None
        self.dw_pre = nans(self.C, self.t) if self.pre else None
        need = self.jz.jz_norm_residual_bwd_workspace_bytes(self.desc)
        self.ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)          # NaN where something is read that nobody wrote
        self.jz.jz_norm_residual_bwd(self.desc, self.y, self.r_out if self.branch else self.r, self.w_post, self.gate, self.w_pre, self.k1, self.k2,
                                     self.dr_out if dr_out == "given" else dr_out, self.dn, self.dr, self.dy, self.dw_post, self.dgate, self.dw_pre, self.ws)
        torch.cuda.synchronize()

    def check_forward(self):
        f = blocks.norm_residual_fwd(*(wide(v) for v in (self.r, self.y, self.w_post, self.gate, self.w_pre)), EPS, RES, BRANCH)
        if self.branch:
            check(self.r_out, f["r_out"], f["mag"], 32, "r_out")
        if self.pre:
            scale = f["rstd_pre"] * np.abs(wide(self.w_pre))
            check(self.n, f["n"], f["mag"] * scale + np.abs(f["n"]), 64, "n")
            # a relative change of r_out's terms changes rstd by mean(r_out * change) rstd^3: where the terms cancel, by more than its own size
            change = f["rstd_pre"] ** 3 * np.mean(np.abs(f["r_out"]) * f["mag"], axis=1, keepdims=True)
            check(self.k2, f["rstd_pre"][:, 0], np.maximum(f["rstd_pre"], change)[:, 0], 64, "rstd_pre")
        if self.k1 is not None:
            check(self.k1, f["rstd_post"][:, 0], f["rstd_post"][:, 0], 32, "rstd_post")

    def check_backward(self, dr_out="given"):
        b = blocks.norm_residual_bwd(wide(self.y), wide(self.r_out if self.branch else self.r), wide(self.w_post), wide(self.gate), wide(self.w_pre),
                                     None if self.k1 is None else wide(self.k1)[:, None], None if self.k2 is None else wide(self.k2)[:, None],
                                     wide(self.dr_out) if dr_out == "given" else dr_out, wide(self.dn), RES, BRANCH, branch=self.branch)
        check(self.dr, b["dr"], b["mag"]["dr"], 128, "dr")
        if self.branch:
            check(self.dy, b["dy"], b["mag"]["dy"], 128, "dy")
        for name in ("dw_post", "dgate", "dw_pre"):
            got = getattr(self, name)
            assert (got is None) == (name not in b)
            if got is not None:
                check(got, b[name], b["mag"][name], 320, name)


@pytest.mark.parametrize("dtype, res", [("f16", None), ("f16", "f32"), ("bf16", None), ("bf16", "f32"), ("f32", None)])
@pytest.mark.parametrize("C", [1, 7, 8, 64, 511, 512, 1000, 1024, 1025, 2048, 4097])
def test_types_and_widths(jz, dtype, res, C):
    c = Case(jz, 19, C, dtype, res)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("C", [4096, 8191, 8192, 8200, 16383, 16384])
@pytest.mark.parametrize("dtype, res", [("f16", "f32"), ("bf16", None)])
def test_wide_rows(jz, dtype, res, C):
    c = Case(jz, 9, C, dtype, res)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 8, 9, 4095, 4096, 4097, 5000])
def test_row_counts(jz, rows):
    c = Case(jz, rows, 200, "f16", "f32")
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("rows, per", [(12, 1), (12, 3), (12, 12), (64, 8), (63, 7), (96, 32), (5000, 1), (5000, 5), (5000, 1000), (5000, 2500), (4608, 9), (4608, 18), (8000, 16)])
@pytest.mark.parametrize("post", [True, False])
def test_gates_of_groups(jz, rows, per, post):
    c = Case(jz, rows, 72, "bf16", "f32", per=per, post=post)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("pre", [True, False])
@pytest.mark.parametrize("dr_out", ["given", None])
def test_parts(jz, post, gate, pre, dr_out):
    if dr_out is None and not pre:
        pytest.skip("no gradient arrives at all")
    c = Case(jz, 50, 328, "f16", post=post, gate=gate, pre=pre)
    c.forward()
    c.check_forward()
    c.backward(dr_out)
    c.check_backward(dr_out)


@pytest.mark.parametrize("dtype, res", [("f16", None), ("bf16", "f32"), ("f32", None)])
def test_the_norm_alone(jz, dtype, res):
    c = Case(jz, 33, 776, dtype, res, branch=False)
    c.forward()
    c.check_forward()
    global RES
    keep, RES = RES, 1.0
    try:
        c.desc.res_scale = 1.0
        c.backward()
        c.check_backward()
    finally:
        RES = keep


def test_in_place(jz):
    a, b = Case(jz, 300, 520, "bf16", "f32"), Case(jz, 300, 520, "bf16", "f32")
    a.forward()
    a.backward()
    b.n, b.k1, b.k2 = nans((300, 520), b.t), nans(300, torch.float32), nans(300, torch.float32)
    jz.jz_norm_residual_fwd(b.desc, b.r, b.y, b.w_post, b.gate, b.w_pre, b.r, b.n, b.k1, b.k2)
    assert torch.equal(a.r_out, b.r) and torch.equal(a.n, b.n)
    dy, dw, dg, dp = torch.empty_like(b.y), nans(520, b.t), nans((1, 520), b.t), nans(520, b.t)
    jz.jz_norm_residual_bwd(b.desc, b.y, b.r, b.w_post, b.gate, b.w_pre, b.k1, b.k2, b.dr_out, b.dn, b.dr_out, dy, dw, dg, dp, a.ws)
    torch.cuda.synchronize()
    for x, y in ((a.dr, b.dr_out), (a.dy, dy), (a.dw_post, dw), (a.dgate, dg), (a.dw_pre, dp)):
        assert torch.equal(x, y)


def test_no_rows_give_zero_parameter_gradients(jz):
    c = Case(jz, 0, 40, "f16")
    c.forward()
    c.backward()
    for v in (c.dw_post, c.dgate, c.dw_pre):
        assert torch.all(v == 0)


def test_rows_of_zeros_and_rows_that_are_not_finite_keep_to_themselves(jz):
    c = Case(jz, 20, 264, "f16", "f32", gate=False)
    c.y[3] = 0
    c.r[3] = 0
    c.y[5, 17] = float("nan")
    c.r[7, 200] = float("inf")
    c.forward()
    assert torch.all(c.r_out[3] == 0) and torch.all(c.n[3] == 0) and abs(float(c.k2[3]) * EPS ** 0.5 - 1) < 1e-5
    assert torch.all(torch.isnan(c.n[5])) and torch.all(torch.isnan(c.r_out[5]))
    assert bool(torch.isinf(c.r_out[7, 200])) and torch.all(torch.isfinite(c.r_out[7, :200]))
    fine = [i for i in range(20) if i not in (5, 7)]
    assert torch.all(torch.isfinite(c.n[fine])) and torch.all(torch.isfinite(c.r_out[fine]))
    c.backward()
    assert torch.all(torch.isfinite(c.dr[fine]))
    fine.remove(3)          # a row of zeros has rstd = 316 twice over: its dy, of the order of 10^5, is outside FP16
    assert torch.all(torch.isfinite(c.dy[fine])) and not torch.any(torch.isnan(c.dy[3]))


def test_same_bits_again_and_in_a_graph(jz):
    c = Case(jz, 3000, 1000, "bf16", per=30)
    c.forward()
    c.backward()
    names = ("r_out", "n", "dr", "dy", "dw_post", "dgate", "dw_pre")
    want = {k: getattr(c, k).clone() for k in names}

    def both():
        jz.jz_norm_residual_fwd(c.desc, c.r, c.y, c.w_post, c.gate, c.w_pre, c.r_out, c.n, c.k1, c.k2)
        jz.jz_norm_residual_bwd(c.desc, c.y, c.r_out, c.w_post, c.gate, c.w_pre, c.k1, c.k2, c.dr_out, c.dn, c.dr, c.dy, c.dw_post, c.dgate, c.dw_pre, c.ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.synchronize()
    assert all(torch.equal(getattr(c, k), want[k]) for k in names)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for _ in range(4):
        for k in names:
            getattr(c, k).fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(c, k), want[k]) for k in names)
        (c.r.float() * 2).sum().item()


def test_gradient_is_the_difference_of_what_the_forward_call_computes(jz):
    """In FP32, along one direction: (f(x + s d) - f(x - s d)) / 2 s.  The loss is a sum of 4096 terms of order one, each within about
    1e-6, so the difference of two losses is within 1e-4 of 64 * 1e-6 / s = 1e-2 relative to gradients of order one: s = 1e-2."""
    c = Case(jz, 32, 128, "f32")
    c.forward()
    c.backward()
    g = np.random.default_rng(99)
    for name, grad in (("r", "dr"), ("y", "dy"), ("w_post", "dw_post"), ("gate", "dgate"), ("w_pre", "dw_pre")):
        base = getattr(c, name)
        d = randn(g, tuple(base.shape), torch.float32)
        slope = float((getattr(c, grad).double() * d.double()).sum())
        loss = []
        for s in (1e-2, -1e-2):
            setattr(c, name, base + s * d)
            c.forward()
            loss.append(float((c.dr_out.double() * c.r_out.double()).sum() + (c.dn.double() * c.n.double()).sum()))
        setattr(c, name, base)
        size = float((getattr(c, grad).double() ** 2).sum() ** 0.5)
        assert abs((loss[0] - loss[1]) / 2e-2 - slope) <= 0.02 * size + 0.02, (name, loss, slope)


@pytest.mark.parametrize("C", [513, 1027, 2049, 4103, 8193])
@pytest.mark.parametrize("post, pre", [(False, False), (True, False), (False, True), (True, True)])
def test_in_place_where_a_row_ends_in_a_wavefront_of_its_own(jz, C, post, pre):
    """The last vector of a row then begins among the elements of another wavefront, which may load them later: the same bits in place as out of place."""
    c = Case(jz, 600, C, per=8, post=post, pre=pre, seed=3)
    c.forward()
    r = c.r.clone()
    n = nans((c.rows, C), c.t) if pre else None
    jz.jz_norm_residual_fwd(c.desc, r, c.y, c.w_post, c.gate, c.w_pre, r, n, c.k1, c.k2)
    torch.cuda.synchronize()
    assert torch.equal(r, c.r_out) and (not pre or torch.equal(n, c.n))
    c.backward()
    dr, dy, dgate = c.dr_out.clone(), torch.empty_like(c.dy), torch.empty_like(c.dgate)
    jz.jz_norm_residual_bwd(c.desc, c.y, c.r_out, c.w_post, c.gate, c.w_pre, c.k1, c.k2, dr, c.dn, dr, dy, c.dw_post, dgate, c.dw_pre, c.ws)
    torch.cuda.synchronize()
    assert torch.equal(dr, c.dr) and torch.equal(dy, c.dy) and torch.equal(dgate, c.dgate)


@pytest.mark.parametrize("rows, per", [(16383, 0), (16384, 0), (16385, 0), (20480, 40), (16384, 128), (2047, 23), (1999, 0), (203, 7)])
def test_slabs_of_many_and_of_few_rows(jz, rows, per):
    c = Case(jz, rows, 72, "bf16", per=per, seed=5)
    c.forward()
    c.backward()
    c.check_forward()
    c.check_backward()
