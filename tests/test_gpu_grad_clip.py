"""jz_grad_norm and jz_grad_clip against their formula in 64 bits.

Tolerances.  Norm: squares and the three additions of eight of them round in FP32, four roundings on the sum at most, halved by the root;
everything else is FP64, and the result rounds once: 2^-24 (4/2 + 1) <= 2^-22 relative.  Output: the factor has the norm's error and one
rounding, the product rounds in FP32 and then to the type: 2^-21 relative besides the type's own rounding."""
import math

import numpy as np
import pytest
import torch

from oracle import blocks
from jzt_blocks import DEV, ROUND, TINY, TYPES, nans, randn, wide

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


class Run:
    def __init__(self, jz, grads, out=None):
        self.jz, self.list = jz, jz.GradList(grads, out)
        need = jz.jz_grad_clip_workspace_bytes(self.list)
        self.ws = torch.full((need,), 0x5a, dtype=torch.uint8, device=DEV)
        self.norm, self.flag = nans(1, torch.float32), torch.full((1,), 77, dtype=torch.int32, device=DEV)
        jz.jz_grad_clip_prepare(self.list, self.ws)

    def clip(self, max_norm, **kw):
        self.jz.jz_grad_clip(self.list, max_norm, self.norm, self.flag, self.ws, **kw)
        torch.cuda.synchronize()
        return float(self.norm.item()), int(self.flag.item())

    def only_norm(self, **kw):
        self.jz.jz_grad_norm(self.list, self.norm, self.flag, self.ws, **kw)
        torch.cuda.synchronize()
        return float(self.norm.item()), int(self.flag.item())


def check_norm(got, exact):
    assert abs(got - exact) <= 2.0 ** -22 * exact, (got, exact)


def check_out(out, g64, c):
    ref = g64 * c
    o = wide(out)
    assert np.all(np.abs(o - ref) <= (ROUND[out.dtype] + 2.0 ** -21) * np.abs(ref) + TINY[out.dtype])


def views(g, sizes, dtype, std, gap=0):
    """Slices of one buffer, one behind the other (gap elements between): they start where their neighbours end."""
    flat = randn(g, (sum(sizes) + gap * len(sizes),), dtype, std)
    at, res = 0, []
    for n in sizes:
        res.append(flat[at:at + n])
        at += n + gap
    return flat, res


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("sizes", [(1,), (3, 0, 7), (16384, 1, 16385), (40001, 255, 2049, 8, 9, 70000), (300000,)])
def test_clip(jz, dtype, in_place, sizes):
    g = np.random.default_rng((3, len(sizes), sizes[0]))
    t = TYPES[dtype]
    flat, grads = views(g, sizes, t, 3.0)
    before = [wide(v) for v in grads]
    out_flat = None if in_place else nans(flat.numel() + 1, t)
    out, at = None, 1                           # outputs start one element off their gradients' places
    if not in_place:
        out = []
        for n in sizes:
            out.append(out_flat[at:at + n])
            at += n
    r = Run(jz, grads, out)
    exact, _, _ = blocks.grad_clip(before, math.inf, 8.0)
    norm, flag = r.only_norm(loss_scale=8.0)
    check_norm(norm, exact)
    assert flag == 0
    assert all(np.array_equal(wide(v), b) for v, b in zip(grads, before))
    for max_norm in (exact * 0.25, exact * 4.0):
        _, _, c = blocks.grad_clip([wide(v) for v in grads], max_norm, 8.0)
        now = [wide(v) for v in grads]
        norm, flag = r.clip(max_norm, loss_scale=8.0)
        check_norm(norm, blocks.grad_clip(now, max_norm, 8.0)[0])
        assert flag == 0
        for o, b in zip(grads if in_place else out, now):
            check_out(o, b, c)
            assert c != 1.0 or np.array_equal(wide(o), b)
    if not in_place:
        assert all(np.array_equal(wide(v), b) for v, b in zip(grads, before))
        assert math.isnan(float(out_flat[0]))


def test_many_tensors_of_mixed_types_and_the_same_bits_again(jz):
    g = np.random.default_rng(5)
    grads = []
    for i in range(300):
        grads.append(randn(g, (int(g.integers(1, 5000)),), list(TYPES.values())[i % 3], 10.0 ** g.uniform(-4, 1)))
    out = [torch.empty_like(v) for v in grads]
    r = Run(jz, grads, out)
    exact, _, c = blocks.grad_clip([wide(v) for v in grads], 1.0, 1.0)
    norm, flag = r.clip(1.0)
    check_norm(norm, exact)
    assert flag == 0 and c < 1.0
    for v, o in zip(grads, out):
        check_out(o, wide(v), c)
    first = [o.clone() for o in out]
    for _ in range(3):
        assert r.clip(1.0) == (norm, 0)
        assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_more_chunks_than_workgroups(jz):
    g = np.random.default_rng(6)
    v = torch.empty(2048 * 16384 + 16384 * 5 + 77, dtype=torch.bfloat16, device=DEV).fill_(0.5)
    v[-1] = 1000.0
    v[123] = -77.0
    r = Run(jz, [v])
    exact = math.sqrt(0.25 * (v.numel() - 2) + 1e6 + 77.0 ** 2)
    norm, flag = r.clip(exact / 2)
    check_norm(norm, exact)
    assert flag == 0
    assert torch.all(v[124:-1] == 0.25) and float(v[-1]) == 500.0 and float(v[123]) == -38.5


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("where", [0, 17, -1])
def test_values_that_are_not_finite(jz, dtype, bad, where):
    g = np.random.default_rng(7)
    v = randn(g, (20011,), TYPES[dtype])
    v[where] = bad
    bits = torch.int32 if dtype == "f32" else torch.int16
    before = v.clone()
    norm, flag = Run(jz, [v]).clip(0.5)
    assert flag == 1 and (math.isnan(norm) if math.isnan(bad) else norm == math.inf)
    assert torch.equal(v.view(bits), before.view(bits))
    out = nans(20011, TYPES[dtype])
    norm, flag = Run(jz, [v], [out]).clip(0.5)
    assert flag == 1 and torch.equal(out.view(bits), before.view(bits))


@pytest.mark.parametrize("dtype, big", [("bf16", 3e38), ("f32", 3e38), ("f16", 65504.0), ("f32", 1e-30), ("bf16", 1e-30), ("f16", 2.0 ** -24)])
def test_squares_outside_the_range_of_fp32(jz, dtype, big):
    v = torch.full((999,), big, dtype=TYPES[dtype], device=DEV)
    x = wide(v)
    out = nans(999, TYPES[dtype])
    exact = math.sqrt(999) * float(x[0])
    norm, flag = Run(jz, [v], [out]).clip(exact / 3 if exact / 3 < 3e38 else 1e38)
    assert flag == 0
    if exact < 3.4e38:
        assert abs(norm - exact) <= 2.0 ** -22 * exact
    else:
        assert norm == math.inf                     # the norm itself is outside FP32; the factor is formed in FP64
    check_out(out, x, (exact / 3 if exact / 3 < 3e38 else 1e38) / exact)


def test_zeros_and_nothing_at_all(jz):
    v = torch.zeros(1000, dtype=torch.float16, device=DEV)
    assert Run(jz, [v]).clip(0.0) == (0.0, 0)
    assert torch.all(v == 0)
    assert Run(jz, []).clip(1.0) == (0.0, 0)
    assert Run(jz, [torch.empty(0, dtype=torch.bfloat16, device=DEV)]).only_norm() == (0.0, 0)
    v.fill_(1.0)
    Run(jz, [v]).clip(0.0)                          # clipped to nothing
    assert torch.all(v == 0)
    v.fill_(1.0)
    norm, flag = Run(jz, [v]).clip(math.inf)
    assert flag == 0 and torch.all(v == 1)


def test_the_scale_on_the_device(jz):
    g = np.random.default_rng(8)
    v = randn(g, (5000,), torch.float16, 20.0)
    state = torch.zeros(2, dtype=torch.int32, device=DEV)
    jz.jz_loss_scale_init(state, 64.0)
    r = Run(jz, [v], [nans(5000, torch.float16)])
    exact, _, c = blocks.grad_clip([wide(v)], 1.0, 64.0)
    norm, flag = r.clip(1.0, state=state, loss_scale=1e30)
    check_norm(norm, exact)
    check_out(r.list.out[0], wide(v), c)


def test_a_table_of_another_list_is_refused_on_the_device(jz):
    v, w = torch.ones(100, device=DEV), torch.ones(100, device=DEV)
    r = Run(jz, [v])
    other = jz.GradList([w])
    for call in (lambda: jz.jz_grad_clip(other, 0.5, r.norm, r.flag, r.ws), lambda: jz.jz_grad_norm(other, r.norm, r.flag, r.ws)):
        r.norm.zero_(), r.flag.zero_()
        call()
        torch.cuda.synchronize()
        assert int(r.flag) == -1 and math.isnan(float(r.norm)) and torch.all(w == 1) and torch.all(v == 1)


def test_on_another_stream_and_in_a_graph(jz):
    g = np.random.default_rng(9)
    v = randn(g, (100003,), torch.bfloat16, 2.0)
    out = nans(100003, torch.bfloat16)
    r = Run(jz, [v], [out])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        jz.jz_grad_clip(r.list, 1.0, r.norm, r.flag, r.ws)
    torch.cuda.synchronize()
    want, norm = out.clone(), float(r.norm)
    check_norm(norm, blocks.grad_clip([wide(v)], 1.0, 1.0)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jz.jz_grad_clip(r.list, 1.0, r.norm, r.flag, r.ws)
    for _ in range(4):
        out.fill_(float("nan"))
        r.norm.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and float(r.norm) == norm and int(r.flag) == 0
        (v.float() * 2).sum().item()                # eager work between the replays


def test_overlaps_are_refused_before_anything_runs(jz):
    v = torch.ones(1000, device=DEV)
    ws = torch.empty(jz.jz_grad_clip_workspace_bytes(jz.GradList([v])) * 4, dtype=torch.uint8, device=DEV)

    def status(grads, out=None, w=ws):
        try:
            jz.jz_grad_clip_prepare(jz.GradList(grads, out), w)
        except jz.JzError as e:
            return e.status
        return jz.JZ_OK
    a, b = v[:500], v[400:900]
    assert status([a, b]) == jz.JZ_ERR_ALIAS                      # in place: written twice
    assert status([a], [v[1:501]]) == jz.JZ_ERR_ALIAS             # not the gradient itself
    assert status([v[:100], v[100:200]], [v[300:400], v[350:450]]) == jz.JZ_ERR_ALIAS
    assert status([v[:100], v[100:200]], [v[100:200], v[:100]]) == jz.JZ_ERR_ALIAS
    assert status([a, b], [torch.empty(500, device=DEV), torch.empty(500, device=DEV)]) == jz.JZ_OK    # read twice is no harm
    assert status([v[:100], v[100:200]], [v[:100], v[300:400]]) == jz.JZ_OK
    assert status([ws[:64].view(torch.float32)]) == jz.JZ_ERR_ALIAS
    assert status([a], None, ws[:64]) == jz.JZ_ERR_WORKSPACE
    assert torch.all(v == 1)


@pytest.mark.parametrize("sizes", [(1572864,), (1572865,), (1572864 - 2049, 2048, 1), (16384 * 90, 16385, 1, 100001, 0, 16383, 8197)])
@pytest.mark.parametrize("dtype", ["f16", "f32"])
def test_lists_of_short_and_of_long_chunks(jz, dtype, sizes):
    g = np.random.default_rng((7, len(sizes), sizes[0]))
    _, grads = views(g, sizes, TYPES[dtype], 0.5)
    before = [wide(v) for v in grads]
    r = Run(jz, grads, None)
    exact, _, _ = blocks.grad_clip(before, math.inf, 4.0)
    _, _, c = blocks.grad_clip(before, exact * 0.125, 4.0)
    norm, flag = r.clip(exact * 0.125, loss_scale=4.0)
    check_norm(norm, exact)
    assert flag == 0
    for o, b in zip(grads, before):
        check_out(o, b, c)
