"""Clipping by the global norm, the norms around a residual block and the gated feed-forward block, in 64 bits (numpy), from their
formulas: what include/jz.h says of jz_grad_clip, jz_norm_residual_fwd / _bwd and jz_ffn_fwd / _bwd.  Test infrastructure only."""
import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


# ---- clipping --------------------------------------------------------------------------------------------------------
def grad_clip(grads, max_norm, scale):
    """(norm, flag, factor): gradients are lists of float64 arrays that carry `scale`."""
    total = 0.0
    bad = False
    for g in grads:
        if not np.all(np.isfinite(g)):
            bad = True
        total += float(np.sum(np.square(g)))
    norm = math.sqrt(total) / scale if not bad else (math.nan if any(np.any(np.isnan(g)) for g in grads) else math.inf)
    return norm, int(bad), max_norm / norm if not bad and norm > max_norm else 1.0


# ---- norms around a block ----------------------------------------------------------------------------------------------
def rstd(v, eps):
    return 1.0 / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps)


def _gate(gate, rows):
    return 1.0 if gate is None else np.repeat(gate, rows // gate.shape[0], axis=0)


def norm_residual_fwd(r, y, w_post, gate, w_pre, eps, res_scale, branch_scale):
    """dict of r_out, n, rstd_post, rstd_pre and, per element, the size of the terms that r_out was added up from (mag)."""
    k1 = None
    if y is None:
        out, mag = r, np.abs(r)
    else:
        p = y
        if w_post is not None:
            k1 = rstd(y, eps)
            p = y * k1 * w_post
        b = branch_scale * _gate(gate, len(r)) * p
        out, mag = res_scale * r + b, np.abs(res_scale * r) + np.abs(b)
    res = dict(r_out=out, rstd_post=k1, mag=mag)
    if w_pre is not None:
        k2 = rstd(out, eps)
        res.update(rstd_pre=k2, n=out * k2 * w_pre)
    return res


def norm_residual_bwd(y, r_out, w_post, gate, w_pre, k1, k2, dr_out, dn, res_scale, branch_scale, branch=True):
    """dict of dr, dy, dw_post, dgate, dw_pre; `mag` holds the sizes of the terms of each.  k1, k2: rstd_post, rstd_pre [rows, 1]."""
    rows = len(r_out if r_out is not None else dr_out)
    R = np.zeros_like(r_out) if dr_out is None else dr_out
    res, mag = {}, {}
    Rm = np.abs(R)
    if dn is not None:
        hat = r_out * k2
        e = w_pre * dn
        c = np.mean(e * hat, axis=1, keepdims=True)
        cm = np.mean(np.abs(e * hat), axis=1, keepdims=True)
        res["dw_pre"], mag["dw_pre"] = np.sum(dn * hat, axis=0), np.sum(np.abs(dn * hat), axis=0)
        R = R + k2 * (e - hat * c)
        Rm = Rm + k2 * (np.abs(e) + np.abs(hat) * cm)
    res["dr"], mag["dr"] = res_scale * R, abs(res_scale) * Rm
    if branch:
        g = _gate(gate, rows)
        dp, dpm = branch_scale * g * R, np.abs(branch_scale * g) * Rm
        yh = None if y is None else y if w_post is None else y * k1
        if gate is not None:
            p = yh if w_post is None else yh * w_post
            per = rows // gate.shape[0]
            res["dgate"] = np.add.reduceat(branch_scale * p * R, np.arange(0, rows, per), axis=0) if rows else np.zeros_like(gate)
            mag["dgate"] = np.add.reduceat(np.abs(branch_scale * p) * Rm, np.arange(0, rows, per), axis=0) if rows else np.zeros_like(gate)
        if w_post is None:
            res["dy"], mag["dy"] = dp, dpm
        else:
            e, em = dp * w_post, dpm * np.abs(w_post)
            res["dw_post"], mag["dw_post"] = np.sum(dp * yh, axis=0), np.sum(dpm * np.abs(yh), axis=0)
            res["dy"] = k1 * (e - yh * np.mean(e * yh, axis=1, keepdims=True))
            mag["dy"] = k1 * (em + np.abs(yh) * np.mean(em * np.abs(yh), axis=1, keepdims=True))
    res["mag"] = mag
    return res


# ---- gated feed-forward block ------------------------------------------------------------------------------------------
def act(kind, v):
    """(act(v), act'(v)) for kind "silu", "gelu" (by the error function), "gelu_tanh", "relu"."""
    if kind == "silu":
        s = np.where(v >= 0, 1.0 / (1.0 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1.0 + np.exp(-np.abs(v))))
        return v * s, s * (1.0 + v * (1.0 - s))
    if kind == "gelu":
        phi = 0.5 * (1.0 + _erf(v / math.sqrt(2.0)))
        return v * phi, phi + v * np.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        k = math.sqrt(2.0 / math.pi)
        t = np.tanh(k * (v + 0.044715 * v ** 3))
        return 0.5 * v * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * v * v)
    assert kind == "relu"
    return np.maximum(v, 0.0), (v > 0).astype(v.dtype)


def ffn_fwd(x, wg, wu, wd, kind):
    g, u = x @ wg.T, x @ wu.T
    h = act(kind, g)[0] * u
    return dict(gate=g, up=u, h=h, y=h @ wd.T)


def ffn_bwd(x, wg, wu, wd, gate, up, h, dy, kind):
    """dx, dwg, dwu, dwd, and the two gradients between (dgate, dup), from the saved gate, up and h."""
    a, da = act(kind, gate)
    dh = dy @ wd
    dg, du = dh * up * da, dh * a
    return dict(dgate=dg, dup=du, dx=dg @ wg + du @ wu, dwg=dg.T @ x, dwu=du.T @ x, dwd=dy.T @ h)
