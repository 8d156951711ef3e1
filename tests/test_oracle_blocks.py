"""The 64-bit formulas of the residual-block operators against differences and by hand (no GPU)."""
import math

import numpy as np
import pytest

from oracle import blocks


def rng(*key):
    return np.random.default_rng(key)


def difference(f, a, at, step=1e-5):
    """(f(a + step) - f(a - step)) / (2 step) in the element `at`; error of the order of step^2."""
    hi, lo = a.copy(), a.copy()
    hi[at] += step
    lo[at] -= step
    return (f(hi) - f(lo)) / (2 * step)


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "relu"])
def test_ffn_gradients_are_the_differences(kind):
    g = rng(1, len(kind))
    M, D, F, O = 3, 4, 5, 6
    t = dict(x=g.standard_normal((M, D)), wg=g.standard_normal((F, D)), wu=g.standard_normal((F, D)), wd=g.standard_normal((O, F)))
    dy = g.standard_normal((M, O))
    f = blocks.ffn_fwd(**t, kind=kind)
    b = blocks.ffn_bwd(**t, gate=f["gate"], up=f["up"], h=f["h"], dy=dy, kind=kind)
    for name in t:
        for at in [(0, 0), (1, 2), tuple(n - 1 for n in t[name].shape)]:
            d = difference(lambda v: float(np.sum(dy * blocks.ffn_fwd(**{**t, name: v}, kind=kind)["y"])), t[name], at)
            assert abs(b["d" + name][at] - d) < 1e-6 * max(1.0, abs(d)), (name, at)


@pytest.mark.parametrize("post, groups, pre", [(True, 2, True), (False, 1, True), (True, 0, False), (False, 0, True), (True, 6, True), (False, 3, False)])
def test_norm_gradients_are_the_differences(post, groups, pre):
    g = rng(2, post, groups, pre)
    M, C = 6, 5
    t = dict(r=g.standard_normal((M, C)), y=g.standard_normal((M, C)), w_post=g.standard_normal(C) if post else None,
             gate=g.standard_normal((groups, C)) if groups else None, w_pre=g.standard_normal(C) if pre else None)
    k = dict(eps=1e-3, res_scale=0.8, branch_scale=1.3)
    dro, dn = g.standard_normal((M, C)), g.standard_normal((M, C)) if pre else None
    f = blocks.norm_residual_fwd(**t, **k)
    b = blocks.norm_residual_bwd(t["y"], f["r_out"], t["w_post"], t["gate"], t["w_pre"], f["rstd_post"], f.get("rstd_pre"), dro, dn, k["res_scale"], k["branch_scale"])

    def loss(**over):
        o = blocks.norm_residual_fwd(**{**t, **over}, **k)
        return float(np.sum(dro * o["r_out"])) + (float(np.sum(dn * o["n"])) if pre else 0.0)
    names = dict(r="dr", y="dy", w_post="dw_post", gate="dgate", w_pre="dw_pre")
    for name, grad in names.items():
        if t[name] is None:
            assert grad not in b
            continue
        for at in [tuple(0 for _ in t[name].shape), tuple(n - 1 for n in t[name].shape)]:
            d = difference(lambda v: loss(**{name: v}), t[name], at)
            assert abs(b[grad][at] - d) < 1e-6 * max(1.0, abs(d)), (name, at)


def test_norm_alone_is_a_vector_of_length_root_channels():
    f = blocks.norm_residual_fwd(np.array([[3.0, 4.0, 0.0, 0.0]]), None, None, None, np.ones(4), 0.0, 1.0, 1.0)
    assert np.allclose(f["n"], np.array([[3.0, 4.0, 0.0, 0.0]]) * 2.0 / 5.0)


def test_clip_by_hand():
    norm, flag, c = blocks.grad_clip([np.array([6.0]), np.array([0.0, 8.0])], 2.5, 2.0)
    assert (norm, flag, c) == (5.0, 0, 0.5)
    assert blocks.grad_clip([np.array([6.0, 8.0])], 5.0, 2.0)[2] == 1.0            # equal: not clipped
    assert blocks.grad_clip([np.zeros(3)], 0.0, 1.0) == (0.0, 0, 1.0)
    assert blocks.grad_clip([np.array([math.inf])], 1.0, 1.0)[1:] == (1, 1.0)
    n, flag, c = blocks.grad_clip([np.array([math.inf, math.nan])], 1.0, 1.0)
    assert math.isnan(n) and flag == 1 and c == 1.0
