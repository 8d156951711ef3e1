"""The 64-bit definitions of the token operators against what they have to be, by other means (no GPU)."""
import numpy as np
import pytest

from oracle import tokens


def test_embedding_gradient_is_the_lookup_s_adjoint():
    g = np.random.default_rng(1)
    ids = g.integers(-2, 13, 40)
    table, dout = g.standard_normal((11, 5)), g.standard_normal((40, 5))
    d, _ = tokens.embed_bwd(ids, dout, 11, 0.7)
    assert np.isclose(np.sum(tokens.embed_fwd(ids, table, 0.7) * dout), np.sum(table * d))
    e = 1e-6
    for v, c in ((0, 0), (3, 4), (10, 2)):
        t = table.copy()
        t[v, c] += e
        slope = np.sum((tokens.embed_fwd(ids, t, 0.7) - tokens.embed_fwd(ids, table, 0.7)) * dout) / e
        assert np.isclose(slope, d[v, c], atol=1e-7)
    more, _ = tokens.embed_bwd(ids, dout, 11, 0.7, before=table)
    assert np.allclose(more, d + table)


@pytest.mark.parametrize("shape", [(6, 9), (9, 6), (7, 7), (1, 5)])
def test_the_iteration_maps_singular_values(shape):
    g = np.random.default_rng(2).standard_normal(shape)
    a, b, c = coefs = (3.4445, -4.7750, 2.0315)
    got, norms = tokens.orthogonalize(g, coefs, 5, 0.0)
    u, s, vt = np.linalg.svd(g / np.linalg.norm(g), full_matrices=False)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert np.allclose(got, (u * s) @ vt) and len(norms) == 6 and np.isclose(norms[-1], np.linalg.norm(s))


def test_muon_without_decay_moves_along_the_iteration_s_result():
    g = np.random.default_rng(3)
    w, v, grad = g.standard_normal((3, 4, 6))
    hp = dict(lr=0.5, momentum=0.9, weight_decay=0.0, update_scale=2.0, nesterov=False)
    w1, v1, o, _ = tokens.muon(w, v, grad, hp, (1.5, -0.5, 0.0), 30, 0.0)
    assert np.allclose(v1, 0.9 * v + grad) and np.allclose(w1, w - o)
    u, _, vt = np.linalg.svd(v1, full_matrices=False)
    assert np.allclose(o, u @ vt)           # these coefficients converge


def test_codes():
    x = np.array([[0.0, 1.0, -127.0, 63.5], [0, 0, 0, 0], [1e-3, 2e-3, np.inf, 0], [0.5, -1.5, 2.5, 127.0]], np.float32)
    q, s = tokens.quantize(x)
    assert q[0].tolist() == [0, 1, -127, 64] and s[0] == 1 and s[1] == 0 and not q[1].any() and np.isnan(s[2]) and not q[2].any()
    assert q[3].tolist() == [0, -2, 2, 127]                     # ties to even
    tiny, s = tokens.quantize(np.array([[190 * 2.0 ** -149, -2.0 ** -149]], np.float32))
    assert s[0] == np.float32(2.0 ** -149) and tiny.tolist() == [[127, -1]]


def test_products_of_codes():
    g = np.random.default_rng(4)
    x, w = g.standard_normal((5, 33)).astype(np.float32), g.standard_normal((7, 33)).astype(np.float32)
    (q, s), (wq, ws) = tokens.quantize(x), tokens.quantize(w)
    y = tokens.linear_i8(q, s, wq, ws)
    step = np.abs(x).max(1)[:, None] / 254 * np.abs(w).sum(1) + np.abs(w).max(1) / 254 * np.abs(x).sum(1)[:, None] + 33 * s[:, None] * ws / 4
    assert np.all(np.abs(y - x.astype(np.float64) @ w.T.astype(np.float64)) <= step)
