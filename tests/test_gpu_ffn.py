"""jz_ffn_fwd and jz_ffn_bwd against their formulas in 64 bits, stage by stage on the tensors that the calls are given and leave.

Tolerances, per element, with u the type's rounding (2^-11, 2^-8) and e = 2^-24:
  gate, up   u |ref| + 8 e sum |x w|: an FP32 sum of K terms in any order is within 8 roundings of sum |terms| (as for the convolutions)
  h          u |ref| + the projections' FP32 error through the formula (|act'| <= 1.13) + 16 e (1 + |gate|) |ref| for exp, reciprocal and products
  y          on the stored h: u |ref| + 8 e sum |h w|
  dx, dw     on the stored gate, up, h: dgate and dup carry one rounding of their own, u of each, through the next product, and FP32's error
  and of every whole result ||out - ref|| / ||ref|| <= 2 u: two roundings of u / sqrt(3) each, and room for the sums."""
import numpy as np
import pytest
import torch

from oracle import blocks
from jzt_blocks import DEV, E32, ROUND, TINY, TYPES, nans, randn, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


ACTS = {"silu": 0, "gelu": 1, "gelu_tanh": 2, "relu": 3}


def strided(t, stride):
    """The same rows, `stride` elements apart in a buffer of NaN."""
    if not stride:
        return t
    rows, cols = t.shape
    flat = torch.full((max(rows, 1) * stride,), float("nan"), dtype=t.dtype, device=DEV)
    v = flat.as_strided((rows, cols), (stride, 1))
    v.copy_(t)
    return v


def close(got, ref, bound, what):
    g = wide(got)
    u = ROUND[got.dtype]
    err = np.abs(g - ref)
    bad = ~(err <= bound + TINY[got.dtype])
    assert not bad.any(), "%s: %d of %d, first at %s: got %r, exact %r, bound %r" % (
        what, bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), g[bad][0], ref[bad][0], np.broadcast_to(bound, ref.shape)[bad][0])
    norm = np.linalg.norm(ref)
    assert np.linalg.norm(g - ref) <= 2 * u * norm + TINY[got.dtype] * ref.size ** 0.5, (what, np.linalg.norm(g - ref) / norm)


class Case:
    def __init__(self, jz, M, D, F, O, dtype="f16", act="silu", strides=(0, 0, 0, 0), seed=0):
        g = np.random.default_rng((M, D, F, O, seed))
        t = TYPES[dtype]
        self.jz, self.t, self.act, self.dims, self.strides = jz, t, act, (M, D, F, O), strides
        self.desc = jz.ffn_desc(M, D, F, O, ACTS[act], jz.dtype_of(t), *strides)
        self.x, self.dy = strided(randn(g, (M, D), t), strides[0]), strided(randn(g, (M, O), t, 0.1), strides[3])
        self.wg, self.wu, self.wd = randn(g, (F, D), t, 1.5 * D ** -0.5), randn(g, (F, D), t, D ** -0.5), randn(g, (O, F), t, F ** -0.5)

    def workspace(self, need, less):
        return torch.full((need - less if less else need,), 0xff, dtype=torch.uint8, device=DEV) if need else None

    def forward(self, keep=True, ws="asked"):
        M, D, F, O = self.dims
        self.h, self.y = nans((M, F), self.t), strided(nans((M, O), self.t), self.strides[1])
        self.gate, self.up = (nans((M, F), self.t), nans((M, F), self.t)) if keep else (None, None)
        ws = self.workspace(self.jz.jz_ffn_fwd_workspace_bytes(self.desc), 0) if ws == "asked" else ws
        self.jz.jz_ffn_fwd(self.desc, self.x, self.wg, self.wu, self.wd, self.h, self.y, self.gate, self.up, ws)
        torch.cuda.synchronize()

    def backward(self, dx=True, weights=True, ws="asked"):
        M, D, F, O = self.dims
        self.dx = strided(nans((M, D), self.t), self.strides[2]) if dx else None
        self.dwg, self.dwu, self.dwd = (nans(s, self.t) for s in ((F, D), (F, D), (O, F))) if weights else (None, None, None)
        ws = self.workspace(self.jz.jz_ffn_bwd_workspace_bytes(self.desc), 0) if ws == "asked" else ws
        self.jz.jz_ffn_bwd(self.desc, self.x if weights else None, self.wg, self.wu, self.wd, self.gate, self.up, self.h if weights else None, self.dy, self.dx,
                           self.dwg, self.dwu, self.dwd, ws)
        torch.cuda.synchronize()

    def check_forward(self):
        u = ROUND[self.t]
        x, wg, wu, wd = (wide(v) for v in (self.x, self.wg, self.wu, self.wd))
        g, up = x @ wg.T, x @ wu.T
        eg, eu = 8 * E32 * (np.abs(x) @ np.abs(wg.T)), 8 * E32 * (np.abs(x) @ np.abs(wu.T))
        if self.gate is not None:
            close(self.gate, g, u * np.abs(g) + 2 * eg, "gate")
            close(self.up, up, u * np.abs(up) + 2 * eu, "up")
        a = blocks.act(self.act, g)[0]
        ref = a * up
        close(self.h, ref, u * np.abs(ref) + 2 * (1.13 * eg * np.abs(up) + np.abs(a) * eu + eg * eu + 16 * E32 * (1 + np.abs(g)) * np.abs(ref)), "h")
        h = wide(self.h)
        ref = h @ wd.T
        close(self.y, ref, u * np.abs(ref) + 16 * E32 * (np.abs(h) @ np.abs(wd.T)), "y")

    def check_backward(self):
        u = ROUND[self.t]
        x, wg, wu, wd, gate, up, h, dy = (wide(v) for v in (self.x, self.wg, self.wu, self.wd, self.gate, self.up, self.h, self.dy))
        b = blocks.ffn_bwd(x, wg, wu, wd, gate, up, h, dy, self.act)
        a, da = blocks.act(self.act, gate)
        edh = 8 * E32 * (np.abs(dy) @ np.abs(wd))
        rel = 16 * E32 * (1 + np.abs(gate)) * np.abs(dy @ wd)
        # absolute, not relative, to the slope: it is a difference of terms up to 1 + |gate|
        eg = u * np.abs(b["dgate"]) + 2 * np.abs(up) * (np.abs(da) * edh + rel) + TINY[self.t]
        eu = u * np.abs(b["dup"]) + 2 * (np.abs(a) * edh + np.abs(gate) * rel) + TINY[self.t]
        if self.dx is not None:
            close(self.dx, b["dx"], u * np.abs(b["dx"]) + 1.1 * (eg @ np.abs(wg) + eu @ np.abs(wu)) + 16 * E32 * (np.abs(b["dgate"]) @ np.abs(wg) + np.abs(b["dup"]) @ np.abs(wu)), "dx")
        if self.dwg is not None:
            for name, ref, e, d in (("dwg", b["dwg"], eg, b["dgate"]), ("dwu", b["dwu"], eu, b["dup"])):
                close(getattr(self, name), ref, u * np.abs(ref) + 1.1 * (e.T @ np.abs(x)) + 16 * E32 * (np.abs(d).T @ np.abs(x)), name)
            close(self.dwd, b["dwd"], u * np.abs(b["dwd"]) + 16 * E32 * (np.abs(dy).T @ np.abs(h)), "dwd")

    def check(self):
        self.forward()
        self.check_forward()
        self.backward()
        self.check_backward()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", list(ACTS))
def test_activations_and_types(jz, dtype, act):
    Case(jz, 70, 96, 136, 80, dtype, act).check()


@pytest.mark.parametrize("M", [1, 2, 3, 7, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_row_counts(jz, M, dtype):
    Case(jz, M, 160, 192, 160, dtype).check()


@pytest.mark.parametrize("D, F, O", [(1, 1, 1), (3, 5, 7), (8, 8, 8), (16, 24, 8), (64, 64, 64), (72, 200, 56), (63, 129, 65), (127, 64, 96), (96, 127, 96), (96, 64, 131),
                                     (250, 334, 250), (264, 328, 520), (1000, 2730, 1000)])
@pytest.mark.parametrize("M", [5, 130])
def test_feature_counts(jz, D, F, O, M):
    Case(jz, M, D, F, O, "bf16" if D % 3 else "f16", "gelu").check()


@pytest.mark.parametrize("M", [1, 24, 150, 520])
@pytest.mark.parametrize("D, F, O", [(256, 512, 256), (512, 1408, 768), (1024, 640, 512), (320, 1088, 576)])
def test_aligned_sizes(jz, M, D, F, O):
    Case(jz, M, D, F, O, "f16", "gelu_tanh").check()
    Case(jz, M, D, F, O, "bf16", "silu").check()


def test_a_large_block(jz):
    Case(jz, 2100, 1024, 2816, 1024, "f16", "silu").check()
    Case(jz, 2048, 768, 2048, 768, "bf16", "silu").check()


@pytest.mark.parametrize("strides", [(200, 0, 0, 0), (0, 168, 0, 0), (0, 0, 104, 0), (0, 0, 0, 256), (137, 99, 101, 97), (104, 104, 104, 104)])
@pytest.mark.parametrize("M", [1, 9, 140])
def test_strides(jz, strides, M):
    c = Case(jz, M, 96, 128, 96, "f16", "silu", strides)
    c.check()
    for v, s in ((c.y, strides[1]), (c.dx, strides[2])):          # nothing between the rows was touched
        if s and M > 1:
            between = v.as_strided((M - 1, s - 96), (s, 1), v.storage_offset() + 96)
            assert torch.all(torch.isnan(between))


@pytest.mark.parametrize("M", [1, 20, 300])
def test_parts_of_the_calls(jz, M):
    c = Case(jz, M, 128, 320, 128, "bf16")
    c.forward()
    c.backward()
    want = dict(y=c.y.clone(), h=c.h.clone(), dx=c.dx.clone(), dwg=c.dwg.clone(), dwu=c.dwu.clone(), dwd=c.dwd.clone())
    gate, up = c.gate, c.up
    c.forward(keep=False)
    assert torch.equal(c.y, want["y"]) and torch.equal(c.h, want["h"])
    c.gate, c.up = gate, up
    c.backward(dx=False)
    assert all(torch.equal(getattr(c, k), want[k]) for k in ("dwg", "dwu", "dwd"))
    c.backward(weights=False)
    assert torch.equal(c.dx, want["dx"])


def test_no_rows(jz):
    c = Case(jz, 0, 64, 96, 64)
    c.forward()
    c.backward()
    for v in (c.dwg, c.dwu, c.dwd):
        assert torch.all(v == 0)


def test_infinities_stay_in_their_rows(jz):
    for M in (9, 200):
        c = Case(jz, M, 128, 256, 128)
        c.x[3, 5] = float("inf")
        c.x[6, 100] = float("nan")
        c.forward()
        fine = [i for i in range(M) if i not in (3, 6)]
        assert torch.all(torch.isfinite(c.y[fine])) and not torch.any(torch.isfinite(c.y[6])) and not torch.all(torch.isfinite(c.y[3]))


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gates_far_from_zero(jz, dtype, act):
    """Activations and slopes at gates up to the type's largest: 0 or the value itself, and no NaN from what overflows on the way."""
    t = TYPES[dtype]
    top = 6e4 if dtype == "f16" else 3e38
    v = [0.0, 1e-7, 1.0, 5.0, 20.0, 31.0, 89.0, 200.0, 3e4, top]
    vals = torch.tensor(v + [-a for a in v], dtype=torch.float64)
    M, D, F = len(vals), 8, 8
    c = Case(jz, M, D, F, 8, dtype, act)
    c.x.zero_(), c.wg.zero_(), c.wu.zero_()
    c.x[:, 0] = vals.to(t).to(DEV)
    c.x[:, 1] = 1.0
    c.wg[:, 0] = 1.0
    c.wu[:, 1] = 0.5
    c.wd.copy_(torch.eye(8, dtype=t))
    c.dy.fill_(1.0)
    c.forward()
    g = wide(c.x[:, :1]) + np.zeros((1, F))
    a, da = blocks.act(act, g)
    assert np.array_equal(wide(c.gate), g)
    u = ROUND[t]
    ok = np.abs(wide(c.h) - 0.5 * a) <= u * np.abs(0.5 * a) + 16 * E32 * (1 + np.abs(g)) * np.abs(0.5 * a) + 1e-30 + TINY[t]
    assert ok.all(), (g[~ok], wide(c.h)[~ok])
    c.backward()
    # dx[:, 0] = sum over the eight hidden units of dy up act'(gate), dx[:, 1] = 0.5 sum of dy act(gate)
    slope = 8 * 0.5 * da[:, 0]
    assert np.all(np.abs(wide(c.dx[:, 0]) - slope) <= 3 * u * np.abs(slope) + 1e-5), (wide(c.dx[:, 0]), slope)
    rest = 8 * 0.5 * a[:, 0]
    fits = np.abs(a[:, 0]) * 4 < top
    assert np.all((np.abs(wide(c.dx[:, 1]) - rest) <= 3 * u * np.abs(rest) + 16 * E32 * (1 + np.abs(g[:, 0])) * np.abs(rest) + 1e-5)[fits])


@pytest.mark.parametrize("M, D, F, O", [(1, 512, 1024, 512), (40, 512, 1024, 512), (1000, 256, 512, 256), (300, 250, 333, 250)])
def test_same_bits_again_on_a_stream_and_in_a_graph(jz, M, D, F, O):
    c = Case(jz, M, D, F, O, "bf16")
    c.forward()
    c.backward()
    names = ("h", "gate", "up", "y", "dx", "dwg", "dwu", "dwd")
    want = {k: getattr(c, k).clone() for k in names}
    need = max(jz.jz_ffn_fwd_workspace_bytes(c.desc), jz.jz_ffn_bwd_workspace_bytes(c.desc))
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device=DEV)

    def both():
        jz.jz_ffn_fwd(c.desc, c.x, c.wg, c.wu, c.wd, c.h, c.y, c.gate, c.up, ws)
        jz.jz_ffn_bwd(c.desc, c.x, c.wg, c.wu, c.wd, c.gate, c.up, c.h, c.dy, c.dx, c.dwg, c.dwu, c.dwd, ws)
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
        (c.x.float() * 2).sum().item()


@pytest.mark.parametrize("M, D, F, O", [(8, 256, 1024, 256), (200, 256, 512, 256), (3000, 128, 256, 128)])
def test_less_workspace_than_reported(jz, M, D, F, O):
    """Fewer splits, other orders of the same sums."""
    c = Case(jz, M, D, F, O, "f16")
    c.forward(ws=None)
    c.check_forward()
    hidden = 2 * ((M * F * 2 + 255) // 256 * 256)
    for spare in (0, 4096, 100000):
        c.backward(ws=torch.full((hidden + spare,), 0xff, dtype=torch.uint8, device=DEV))
        c.check_backward()


@pytest.mark.parametrize("M, D, F, O", [(70, 101, 203, 99), (300, 250, 333, 250), (300, 256, 333, 256), (300, 255, 512, 256), (300, 256, 512, 255), (777, 1001, 2731, 1001)])
@pytest.mark.parametrize("strides", [(0, 0, 0, 0), (1037, 1041, 1029, 1055)])
def test_rows_that_are_not_on_16_bytes(jz, M, D, F, O, strides):
    """With copies of the operands in the workspace, and where it has no room for them."""
    c = Case(jz, M, D, F, O, "bf16", "silu", strides)
    c.check()
    c.forward(ws=None)
    c.check_forward()
    c.backward(ws=torch.full((2 * ((M * ((F + 7) // 8 * 8) * 2 + 255) // 256 * 256),), 0xff, dtype=torch.uint8, device=DEV))
    c.check_backward()


def test_gradient_is_the_difference(jz):
    """The loss sum(dy y) of the 64-bit formula at the same inputs, by differences, against the kernels' gradients along one direction of each input:
    the gradients are within 2 u of the formula's (the bound of every whole result), the difference within 1e-6 of it."""
    c = Case(jz, 40, 72, 104, 56, "f16", "gelu")
    c.forward()
    c.backward()
    t = dict(x=wide(c.x), wg=wide(c.wg), wu=wide(c.wu), wd=wide(c.wd))
    dy = wide(c.dy)
    g = np.random.default_rng(12)
    for name in t:
        d = g.standard_normal(t[name].shape)
        s = 1e-5
        up, down = (float(np.sum(dy * blocks.ffn_fwd(**{**t, name: t[name] + k * s * d}, kind="gelu")["y"])) for k in (1, -1))
        got = wide(getattr(c, "d" + name))
        assert abs((up - down) / (2 * s) - float(np.sum(got * d))) <= 4 * 2.0 ** -11 * np.linalg.norm(got) * np.linalg.norm(d) + 1e-6, name
