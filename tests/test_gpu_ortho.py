"""Orthogonalised updates against the iteration in 64 bits.

How far a result may be off, in the 2-norm of all elements, relative to the result's: a step leaves its product with independent errors of relative size 2^-23 of its terms
(22-bit parts, the product of two low parts left out) and its FP32 sums with less than 2^-19 at the lengths here; through B = a I + b A + c A^2 an error of A counts at most
|b| + 2 |c| |A| < 11 times, one of B as |X|: together less than eta = 2^-18 |X|.  The steps that follow take it on at most 3.9 times each (the largest slope of the polynomial where its
values live, up to 1.21).  With the iterates' own norms: sum over steps k of 3.9^(steps - k) eta |X_k| / |X_steps|, and the result's own rounding."""
import numpy as np
import pytest
import torch

from jzt_blocks import DEV, E32, ROUND, TYPES, check, nans, randn, wide
from oracle import tokens

pytestmark = pytest.mark.gpu
COEFS, EPS = (3.4445, -4.7750, 2.0315), 1e-7
C32 = tuple(float(np.float32(c)) for c in COEFS)


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


def allowed(norms):
    steps = len(norms) - 1
    return sum(3.9 ** (steps - k) * 2.0 ** -18 * norms[k] for k in range(steps + 1)) / norms[-1]


def matrices(g, B, R, C, dtype, scale=1.0):
    """A few strong directions over noise."""
    k = max(1, min(4, R, C))
    x = g.standard_normal((B, R, C)) * 0.3 + g.standard_normal((B, R, k)) @ g.standard_normal((B, k, C))
    return torch.from_numpy(x * scale).to(dtype).to(DEV)


def run(jz, x, out, steps=5, coefs=COEFS, eps=EPS, stride=0, y=None):
    B, R, C = x.shape
    d = jz.ortho_desc(B, R, C, jz.dtype_of(x.dtype), jz.dtype_of(out), steps, coefs, eps, stride)
    ws = torch.full((jz.jz_orthogonalize_workspace_bytes(d),), 0x7f, dtype=torch.uint8, device=DEV)
    y = nans((B, R, C), out) if y is None else y
    jz.jz_orthogonalize(d, x, y, ws)
    torch.cuda.synchronize()
    return y


def against(y, x, steps=5, coefs=C32, eps=float(np.float32(EPS))):
    for got, m in zip(wide(y), wide(x)):
        ref, norms = tokens.orthogonalize(m, coefs, steps, eps)
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert off <= allowed(norms) + ROUND[y.dtype], (off, allowed(norms))


SIZES = [(1, 1, 1), (2, 1, 9), (1, 9, 1), (3, 5, 7), (1, 32, 32), (2, 33, 31), (1, 64, 200), (1, 200, 64), (4, 65, 130), (1, 129, 128), (2, 100, 333), (1, 333, 100), (1, 300, 300), (40, 96, 40),
         (1, 64, 1500)]


@pytest.mark.parametrize("types", [("f16", "f16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("B,R,C", SIZES)
def test_against_64_bits(jz, types, B, R, C):
    g = np.random.default_rng([1, B, R, C])
    x = matrices(g, B, R, C, TYPES[types[0]])
    against(run(jz, x, TYPES[types[1]]), x)


@pytest.mark.parametrize("B,R,C", [(1, 640, 1100), (3, 700, 500), (8, 512, 512), (1, 1500, 1400), (26, 300, 260)])
def test_larger_tiles(jz, B, R, C):
    g = np.random.default_rng([2, B, R, C])
    x = matrices(g, B, R, C, torch.float32)
    against(run(jz, x, torch.float32), x)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("B,R,C", [(3, 100, 140), (5, 31, 33), (2, 150, 260), (3, 260, 150), (2, 140, 1400), (1, 600, 590)])
def test_bf16_results(jz, steps, B, R, C):
    """The operands of the last product rounded to FP16, 2^-12 each: with BF16's own rounding, half a step at most and a third of its square on average, below half a step."""
    g = np.random.default_rng([12, steps, B, R, C])
    x = matrices(g, B, R, C, torch.float32)
    against(run(jz, x, torch.bfloat16, steps=steps), x, steps=steps)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("B,R,C", [(16, 900, 880), (1, 2700, 2690)])
def test_tiles_of_192(jz, B, R, C, out):
    """Symmetric products (the first) and the last one (the second) of the size for which neither 256 nor 128 fill the chip."""
    g = np.random.default_rng([9, B, R, C])
    x = matrices(g, B, R, C, torch.bfloat16)
    against(run(jz, x, TYPES[out], steps=2), x, steps=2)


@pytest.mark.parametrize("B,R,C", [(1, 20, 9000), (16, 2693, 80), (2, 31000, 5), (3, 100, 777), (600, 33, 70), (1, 128, 4103)])
def test_narrow_ones(jz, B, R, C):
    """Long sums that several workgroups share, and many short ones; in the same order every time."""
    g = np.random.default_rng([8, B, R, C])
    x = matrices(g, B, R, C, torch.bfloat16)
    y = run(jz, x, torch.float32)
    against(y, x)
    assert torch.equal(y, run(jz, x, torch.float32))


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_steps_and_coefficients(jz, steps):
    g = np.random.default_rng(3)
    x = matrices(g, 2, 50, 70, torch.float32)
    against(run(jz, x, torch.float32, steps), x, steps)
    y = run(jz, x, torch.float32, steps, (1.5, -0.5, 0.0), 0.0)
    against(y, x, steps, (1.5, -0.5, 0.0), 0.0)
    if steps == 8:
        s = np.linalg.svd(wide(run(jz, x, torch.float32, 24, (1.5, -0.5, 0.0), 0.0))[0], compute_uv=False)
        assert np.all(np.abs(s - 1) <= 1e-4)                    # these converge


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e4, 1e25])
def test_sizes_of_the_elements(jz, scale):
    """The sum of squares leaves FP32's range; the result does not depend on the factor but through eps."""
    g = np.random.default_rng(4)
    x = matrices(g, 2, 40, 48, torch.float32, scale)
    against(run(jz, x, torch.float32, eps=0.0), x, eps=0.0)


def test_zeros_and_matrices_that_are_not_finite(jz):
    g = np.random.default_rng(5)
    x = matrices(g, 5, 36, 70, torch.float16)
    x[1] = 0
    x[2, 3, 5] = float("inf")
    x[4, 35, 69] = float("nan")
    for eps in (EPS, 0.0):
        y = run(jz, x, torch.float16, eps=eps)
        assert bool((y[1] == 0).all()) and bool(torch.isnan(y[[2, 4]]).all())
        against(y[[0, 3]], x[[0, 3]])


@pytest.mark.parametrize("R,C", [(100, 140), (100, 400), (300, 70)])
@pytest.mark.parametrize("steps", [1, 3, 5, 6, 7])
def test_matrices_of_low_rank(jz, R, C, steps):
    """Where a matrix has nothing the polynomial is a^steps; what rounding left there grows by as much."""
    g = np.random.default_rng(6)
    x = torch.from_numpy(g.standard_normal((1, R, 3)) @ g.standard_normal((1, 3, C))).float().to(DEV)
    against(run(jz, x, torch.float32, steps), x, steps)


def test_strided_batch(jz):
    g = np.random.default_rng(7)
    B, R, C, stride = 3, 40, 56, 40 * 56 + 24
    room = torch.full((B * stride,), 9.0, dtype=torch.float32, device=DEV)
    x = room.as_strided((B, R, C), (stride, C, 1))
    x.copy_(matrices(g, B, R, C, torch.float32))
    out = torch.full((B * stride,), 3.0, dtype=torch.bfloat16, device=DEV)
    y = run(jz, x, torch.bfloat16, stride=stride, y=out.as_strided((B, R, C), (stride, C, 1)))
    against(y, x)
    assert bool((out.view(B, stride)[:, R * C:] == 3).all()) and bool((room.view(B, stride)[:, R * C:] == 9).all())


HP = dict(lr=0.05, momentum=0.9, weight_decay=0.02, update_scale=1.3, nesterov=True)


def muon_state(g, B, R, C, dtype, S):
    grad = matrices(g, B, R, C, dtype, 1e-2 * S)
    return dict(grad16=grad, momentum=matrices(g, B, R, C, torch.float32, 3e-2), master=randn(g, (B, R, C), torch.float32, 0.1), weight16=nans((B, R, C), dtype))


def muon(jz, s, hp, S, state=None, skip=None, flag=None, stream=None, stride=0):
    B, R, C = s["grad16"].shape
    d = jz.ortho_desc(B, R, C, jz.dtype_of(s["grad16"].dtype), coefs=COEFS, eps=EPS, stride=stride)
    ws = torch.full((jz.jz_muon_mp_update_workspace_bytes(d),), 0x7f, dtype=torch.uint8, device=DEV)
    flag = torch.full((1,), 77, dtype=torch.int32, device=DEV) if flag is None else flag
    jz.jz_muon_mp_update(d, jz.muon_hparams(**hp, loss_scale=S), s["master"], s["momentum"], s["grad16"], s["weight16"], flag, ws, state, skip, stream)
    torch.cuda.synchronize()
    return int(flag)


def check_muon(s, before, hp, S):
    h = {k: float(np.float32(v)) if not isinstance(v, bool) else v for k, v in hp.items()}
    for i in range(len(s["master"])):
        w0, v0, g0 = wide(before["master"][i]), wide(before["momentum"][i]), wide(before["grad16"][i]) / S
        w, v, o, norms = tokens.muon(w0, v0, g0, h, C32, 5, float(np.float32(EPS)))
        mag = np.abs(h["momentum"] * v0) + np.abs(g0)
        # the gradient's factor, the product, the sum
        check(s["momentum"][i], v, mag, 3, "momentum")
        # the iteration's result as a whole, then decay, scale, sum, rate and difference by element
        got = wide(s["master"][i])
        off = h["lr"] * h["update_scale"] * allowed(norms) * np.linalg.norm(o)
        rest = 6 * E32 * (np.abs(w0) + h["lr"] * (np.abs(h["update_scale"] * o) + np.abs(h["weight_decay"] * w0)))
        # u has three roundings itself, which the iteration takes on as it does its first step's
        assert np.linalg.norm(got - w) <= off + np.linalg.norm(rest)
        assert torch.equal(s["weight16"][i], s["master"][i].to(s["weight16"].dtype))


@pytest.mark.parametrize("B,R,C", [(1, 64, 96), (3, 70, 33), (2, 1, 40), (5, 130, 129), (12, 256, 320)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("nesterov", [True, False])
def test_update(jz, B, R, C, dtype, nesterov):
    g = np.random.default_rng([8, B, R, C])
    S, hp = 512.0, dict(HP, nesterov=nesterov)
    s = muon_state(g, B, R, C, TYPES[dtype], S)
    for _ in range(2):
        before = {k: v.clone() for k, v in s.items()}
        assert muon(jz, s, hp, S) == 0
        check_muon(s, before, hp, S)
        assert torch.equal(s["grad16"], before["grad16"])


def test_the_scale_on_the_device(jz):
    g = np.random.default_rng(9)
    a = muon_state(g, 2, 50, 60, torch.float16, 256.0)
    b = {k: v.clone() for k, v in a.items()}
    state = torch.zeros(2, dtype=torch.int32, device=DEV)
    jz.jz_loss_scale_init(state, 256.0)
    assert muon(jz, a, HP, 256.0) == muon(jz, b, HP, -1.0, state) == 0
    assert all(torch.equal(a[k], b[k]) for k in ("master", "momentum", "weight16"))
    assert jz.loss_scale_state(state) == (256.0, 0)


@pytest.mark.parametrize("how", ["inf", "nan", "skip"])
def test_an_overflow_leaves_everything(jz, how):
    g = np.random.default_rng(10)
    s = muon_state(g, 3, 40, 90, torch.float16, 64.0)
    if how != "skip":
        s["grad16"][2, 39, 89] = float(how)
    before = {k: v.clone() for k, v in s.items()}
    skip = torch.full((1,), int(how == "skip"), dtype=torch.int32, device=DEV)
    assert muon(jz, s, HP, 64.0, skip=skip) == 1
    for k in s:
        assert torch.equal(s[k].view(torch.int16 if s[k].element_size() == 2 else torch.int32), before[k].view(torch.int16 if s[k].element_size() == 2 else torch.int32)), k
    skip.zero_()
    s["grad16"] = before["grad16"] = muon_state(g, 3, 40, 90, torch.float16, 64.0)["grad16"]
    assert muon(jz, s, HP, 64.0, skip=skip) == 0
    check_muon(s, before, HP, 64.0)


@pytest.mark.parametrize("how", ["inf", "skip"])
def test_an_overflow_of_many_sums(jz, how):
    """More partial sums than a workgroup adds up by itself."""
    g = np.random.default_rng(11)
    s = muon_state(g, 2, 2100, 2050, torch.float16, 64.0)
    x = float(s["grad16"][1, 7, 2049])
    if how != "skip":
        s["grad16"][1, 7, 2049] = float(how)
    before = {k: v.clone() for k, v in s.items()}
    skip = torch.full((1,), int(how == "skip"), dtype=torch.int32, device=DEV)
    assert muon(jz, s, HP, 64.0, skip=skip) == 1
    for k in ("momentum", "master"):
        assert torch.equal(s[k], before[k]), k
    assert bool(torch.isnan(s["weight16"]).all())
    skip.zero_()
    s["grad16"][1, 7, 2049] = x
    assert muon(jz, s, HP, 64.0, skip=skip) == 0
    assert torch.equal(s["weight16"], s["master"].half()) and bool((s["master"] != before["master"]).any(2).all())


def test_without_matrices(jz):
    d = jz.ortho_desc(0, 8, 8)
    e, f = torch.empty((0, 8, 8), dtype=torch.float16, device=DEV), torch.empty((0, 8, 8), device=DEV)
    flag, skip = torch.full((1,), 5, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    jz.jz_orthogonalize(d, e, e, None)
    ws = torch.empty(max(16, jz.jz_muon_mp_update_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    jz.jz_muon_mp_update(d, jz.muon_hparams(), f, f, e, e, flag, ws)
    assert int(flag) == 0
    jz.jz_muon_mp_update(d, jz.muon_hparams(), f, f, e, e, flag, ws, skip=skip)
    assert int(flag) == 1


def test_in_a_graph_and_on_another_stream(jz):
    g = np.random.default_rng(11)
    a = muon_state(g, 4, 72, 100, torch.float16, 64.0)
    b = {k: v.clone() for k, v in a.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert muon(jz, a, HP, 64.0, stream=side) == muon(jz, b, HP, 64.0) == 0
    assert all(torch.equal(a[k], b[k]) for k in a)
    d = jz.ortho_desc(4, 72, 100, coefs=COEFS, eps=EPS)
    ws, flag = torch.empty(jz.jz_muon_mp_update_workspace_bytes(d), dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    hp = jz.muon_hparams(**HP, loss_scale=64.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jz.jz_muon_mp_update(d, hp, b["master"], b["momentum"], b["grad16"], b["weight16"], flag, ws)
    for _ in range(4):
        new = muon_state(g, 4, 72, 100, torch.float16, 64.0)["grad16"]
        a["grad16"].copy_(new)
        b["grad16"].copy_(new)
        muon(jz, a, HP, 64.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for k in a) and int(flag) == 0
