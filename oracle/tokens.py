"""Embedding lookup and its gradient, orthogonalised updates and products in 8-bit integers, in 64 bits (numpy), from their formulas: what include/jz.h says of
jz_embed_fwd / _bwd, jz_orthogonalize, jz_muon_mp_update, jz_quantize_i8, jz_linear_i8 and jz_ffn_i8_fwd.  Test infrastructure only."""
import numpy as np

from .blocks import act


# ---- embedding --------------------------------------------------------------------------------------------------------
def embed_fwd(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    there = (ids >= 0) & (ids < len(table))
    out[there] = table[ids[there]] * scale
    return out


def embed_bwd(ids, dout, vocab, scale, before=None):
    """(gradient, size of the terms of each element times the roundings of their sum): n terms, the scale, and what was there."""
    there = np.nonzero((ids >= 0) & (ids < vocab))[0]
    d, mag = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1]))
    np.add.at(d, ids[there], dout[there])
    np.add.at(mag, ids[there], np.abs(dout[there]))
    count = np.bincount(ids[there], minlength=vocab)[:, None]
    d, mag = d * scale, mag * abs(scale)
    if before is not None:
        d, mag = d + before, mag + np.abs(before)
    return d, mag * (count + 2)


# ---- orthogonalisation --------------------------------------------------------------------------------------------------
def orthogonalize(g, coefs, steps, eps):
    """(result, the norms of the iterates) of one matrix."""
    a, b, c = coefs
    x = g / (np.linalg.norm(g) + eps) if np.linalg.norm(g) + eps > 0 else g
    tall = g.shape[0] > g.shape[1]
    if tall:
        x = x.T
    norms = [np.linalg.norm(x)]
    for _ in range(steps):
        A = x @ x.T
        x = a * x + (b * A + c * (A @ A)) @ x
        norms.append(np.linalg.norm(x))
    return (x.T if tall else x), norms


def muon(w, v, g, hp, coefs, steps, eps):
    """(weights, momentum, result of the iteration, norms of the iterates) of one matrix; hp: dict of jz_muon_hparams."""
    v = hp["momentum"] * v + g
    o, norms = orthogonalize(g + hp["momentum"] * v if hp["nesterov"] else v, coefs, steps, eps)
    return w - hp["lr"] * (hp["update_scale"] * o + hp["weight_decay"] * w), v, o, norms


# ---- 8-bit integers -------------------------------------------------------------------------------------------------------
def quantize(x):
    """(codes, scales) of the rows of x (FP32 values): two FP32 divisions, as the definition has them."""
    x = np.asarray(x, np.float32)
    most = np.max(np.abs(x), axis=1)
    bad = ~np.isfinite(x).all(axis=1)
    with np.errstate(all="ignore"):
        s = (most / np.float32(127.0)).astype(np.float32)
        q = np.rint(x / np.where(s > 0, s, np.float32(1.0))[:, None])
    q = np.where((s > 0)[:, None] & ~bad[:, None], np.clip(q, -127, 127), 0)
    return q.astype(np.int8), np.where(bad, np.float32(np.nan), s)


def linear_i8(q, s, wq, ws):
    return (q.astype(np.int64) @ wq.astype(np.int64).T) * (s.astype(np.float64)[:, None] * ws.astype(np.float64))


def ffn_i8(q, s, gate, up, down, kind):
    """(y, how far it may be from it: the codes of h that lie so near a border that FP32 may have the neighbour, and the error of h's largest value).  gate, up, down:
    (codes, scales)."""
    g, u = linear_i8(q, s, *gate), linear_i8(q, s, *up)
    h = act(kind, g)[0] * u
    # roundings of FP32 behind h: three of each projection, the activation's own (10 (1 + |g|)), what it makes of g's (1 + |g|), the product
    off = (16 + 16 * np.abs(g)) * 2.0 ** -24
    qh, sh = quantize(h)
    with np.errstate(all="ignore"):
        t = np.abs(h / np.where(sh > 0, sh, 1.0)[:, None].astype(np.float64))
        worst = np.max(off, axis=1, keepdims=True) + off + 2.0 ** -23
        near = np.abs(t - np.floor(t) - 0.5) <= t * worst
    y = linear_i8(qh, sh, *down)
    flips = (near.astype(np.float64) @ np.abs(down[0].astype(np.float64)).T) * (sh.astype(np.float64)[:, None] * down[1].astype(np.float64))
    return y, flips + np.abs(y) * worst.max(axis=1, keepdims=True)
