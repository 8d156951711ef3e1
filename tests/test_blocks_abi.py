"""Refusals of the residual-block entry points, found on the host before anything is launched (no GPU needed)."""
import ctypes
import math

import numpy as np
import pytest

A = 0x10000000      # an address that is never followed: every call here is refused, or has nothing to do


@pytest.fixture(scope="module")
def jz():
    import os

    from paper_1807_11205_amd import api
    if not os.path.exists(api.LIB_PATH):
        from paper_1807_11205_amd import build
        build.build()
    return api


def grad_list(jz, addresses, numel, dtypes, out=None):
    p, n, t = np.array(addresses, np.uint64), np.array(numel, np.int64), np.array(dtypes, np.int32)
    o = None if out is None else np.array(out, np.uint64)
    c = jz.jz_grad_list(len(p), p.ctypes.data, None if o is None else o.ctypes.data, n.ctypes.data, t.ctypes.data)
    c._keep = (p, n, t, o)
    return c


def test_grad_list_checks(jz):
    L, n = jz.lib(), ctypes.c_size_t(0)

    def size(c):
        return L.jz_grad_clip_workspace_bytes(ctypes.byref(c), ctypes.byref(n))
    assert size(grad_list(jz, [A, A + 64], [16, 8], [0, 2])) == jz.JZ_OK and n.value > 0
    small = n.value
    assert size(grad_list(jz, [A], [1 << 30], [1])) == jz.JZ_OK and n.value > small
    assert size(grad_list(jz, [], [], [])) == jz.JZ_OK and n.value > 0
    assert size(grad_list(jz, [0], [0], [0])) == jz.JZ_OK                      # an empty tensor has no address
    assert size(grad_list(jz, [0], [1], [0])) == jz.JZ_ERR_NULL
    assert size(grad_list(jz, [A], [4], [0], out=[0])) == jz.JZ_ERR_NULL
    assert size(grad_list(jz, [A], [-1], [0])) == jz.JZ_ERR_SHAPE
    assert size(grad_list(jz, [A], [1], [3])) == jz.JZ_ERR_SHAPE
    assert size(grad_list(jz, [A + 1], [1], [0])) == jz.JZ_ERR_ALIGN
    assert size(grad_list(jz, [A + 2], [1], [2])) == jz.JZ_ERR_ALIGN
    assert size(grad_list(jz, [A + 2], [1], [0])) == jz.JZ_OK                  # its own elements' alignment is enough
    assert size(grad_list(jz, [A], [1 << 50], [0])) == jz.JZ_ERR_UNSUPPORTED
    bad = grad_list(jz, [A], [1], [0])
    bad.num_tensors = -1
    assert size(bad) == jz.JZ_ERR_SHAPE
    bad.num_tensors, bad.dtypes = 1, None
    assert size(bad) == jz.JZ_ERR_NULL
    assert L.jz_grad_clip_workspace_bytes(None, ctypes.byref(n)) == jz.JZ_ERR_NULL
    assert L.jz_grad_clip_workspace_bytes(ctypes.byref(bad), None) == jz.JZ_ERR_NULL


def test_clip_checks(jz):
    L, n = jz.lib(), ctypes.c_size_t(0)
    c = grad_list(jz, [A], [1000], [0])
    assert L.jz_grad_clip_workspace_bytes(ctypes.byref(c), ctypes.byref(n)) == jz.JZ_OK
    ws, norm, flag = A + (1 << 20), A + (1 << 21), A + (1 << 21) + 8

    def clip(max_norm=1.0, scale=1.0, state=None, norm=norm, flag=flag, ws=ws, size=n.value, c=c):
        return L.jz_grad_clip(ctypes.byref(c), max_norm, scale, state, norm, flag, ws, size, None)
    assert clip(max_norm=-1.0) == jz.JZ_ERR_SHAPE and clip(max_norm=math.nan) == jz.JZ_ERR_SHAPE
    assert clip(scale=0.0) == clip(scale=-2.0) == clip(scale=math.inf) == clip(scale=math.nan) == jz.JZ_ERR_SHAPE
    assert clip(norm=None) == clip(flag=None) == jz.JZ_ERR_NULL
    assert clip(ws=None) == clip(size=n.value - 1) == jz.JZ_ERR_WORKSPACE
    assert clip(ws=ws + 8) == clip(norm=norm + 2) == clip(flag=flag + 1) == clip(state=A + 4) == jz.JZ_ERR_ALIGN
    assert clip(norm=ws + 16) == clip(flag=ws + n.value - 4) == clip(flag=norm) == clip(state=norm) == clip(state=ws) == jz.JZ_ERR_ALIAS
    assert L.jz_grad_norm(ctypes.byref(c), 0.0, None, norm, flag, ws, n.value, None) == jz.JZ_ERR_SHAPE
    assert L.jz_grad_norm(None, 1.0, None, norm, flag, ws, n.value, None) == jz.JZ_ERR_NULL
    assert L.jz_grad_clip_prepare(ctypes.byref(c), None, n.value, None) == jz.JZ_ERR_WORKSPACE
    assert L.jz_grad_clip_prepare(ctypes.byref(c), ws, n.value - 1, None) == jz.JZ_ERR_WORKSPACE
    assert L.jz_grad_clip_prepare(ctypes.byref(c), ws + 4, n.value, None) == jz.JZ_ERR_ALIGN
    assert L.jz_grad_clip_prepare(ctypes.byref(grad_list(jz, [A, A + 100], [1000, 8], [0, 0])), ws, n.value, None) == jz.JZ_ERR_ALIAS


def norm_call(jz, forward=True, ws_bytes=None, **over):
    d = jz.norm_residual_desc(16, 64, 0, 0, 0)
    for k in list(over):
        if hasattr(d, k):
            setattr(d, k, over.pop(k))
    at = {k: A + i * (1 << 20) for i, k in enumerate(["r", "y", "w_post", "gate", "w_pre", "r_out", "n", "rstd_post", "rstd_pre", "dr_out", "dn", "dr", "dy",
                                                      "dw_post", "dgate", "dw_pre", "ws"])}
    at.update(over)
    names = ["r", "y", "w_post", "gate", "w_pre", "r_out", "n", "rstd_post", "rstd_pre"]
    if forward:
        return jz.lib().jz_norm_residual_fwd(ctypes.byref(d), *(at[k] for k in names), None)
    n = ctypes.c_size_t(0)
    jz.lib().jz_norm_residual_bwd_workspace_bytes(ctypes.byref(d), ctypes.byref(n))
    names = ["y", "r_out", "w_post", "gate", "w_pre", "rstd_post", "rstd_pre", "dr_out", "dn", "dr", "dy", "dw_post", "dgate", "dw_pre", "ws"]
    return jz.lib().jz_norm_residual_bwd(ctypes.byref(d), *(at[k] for k in names), n.value if ws_bytes is None else ws_bytes, None)


@pytest.mark.parametrize("forward", [True, False])
def test_norm_descriptors(jz, forward):
    for bad in (dict(rows=-1), dict(channels=0), dict(channels=-8), dict(rows_per_group=-1), dict(rows_per_group=5), dict(dtype=3), dict(dtype=-1),
                dict(res_dtype=7), dict(eps=-1.0), dict(eps=math.nan), dict(res_scale=math.inf), dict(branch_scale=math.nan)):
        assert norm_call(jz, forward, **bad) == jz.JZ_ERR_SHAPE, bad
    for bad in (dict(res_dtype=1), dict(dtype=1, res_dtype=0), dict(dtype=2, res_dtype=0), dict(channels=16385), dict(rows=1 << 31)):
        assert norm_call(jz, forward, **bad) == jz.JZ_ERR_UNSUPPORTED, bad


def test_norm_forward_arguments(jz):
    for bad in (dict(r=None), dict(y=None), dict(w_pre=None), dict(rstd_pre=None), dict(rstd_post=None), dict(r_out=None), dict(r_out=None, n=None),
                dict(r_out=None, w_post=None)):
        assert norm_call(jz, True, **bad) == jz.JZ_ERR_NULL, bad
    for k in ("r", "y", "w_post", "gate", "w_pre", "r_out", "n", "rstd_post", "rstd_pre"):
        assert norm_call(jz, True, **{k: A + (40 << 20) + 8}) == jz.JZ_ERR_ALIGN, k
    for bad in (dict(n=A), dict(r_out=A + 16), dict(n=A + (1 << 20) + 1024), dict(rstd_pre=A + (7 << 20)), dict(r_out=A + (6 << 20) + 512)):
        assert norm_call(jz, True, **bad) == jz.JZ_ERR_ALIAS, bad
    assert norm_call(jz, True, rows=0) == jz.JZ_OK


def test_norm_backward_arguments(jz):
    for bad in (dict(dr=None), dict(dy=None), dict(y=None), dict(r_out=None), dict(w_pre=None), dict(rstd_pre=None), dict(rstd_post=None), dict(dw_post=None),
                dict(dgate=None), dict(dw_pre=None), dict(dn=None, dr_out=None)):
        assert norm_call(jz, False, **bad) == jz.JZ_ERR_NULL, bad
    for k in ("y", "r_out", "w_post", "gate", "w_pre", "rstd_post", "rstd_pre", "dr_out", "dn", "dr", "dy", "dw_post", "dgate", "dw_pre", "ws"):
        assert norm_call(jz, False, **{k: A + (40 << 20) + 8}) == jz.JZ_ERR_ALIGN, k
    for bad in (dict(dr=A + (9 << 20) + 16), dict(dy=A + (1 << 20)), dict(dw_pre=A + (13 << 20)), dict(ws=A + (9 << 20)), dict(dgate=A + (16 << 20))):
        assert norm_call(jz, False, **bad) == jz.JZ_ERR_ALIAS, bad
    assert norm_call(jz, False, ws=None) == norm_call(jz, False, ws_bytes=16) == jz.JZ_ERR_WORKSPACE


def ffn_call(jz, forward=True, ws_bytes=None, **over):
    d = jz.ffn_desc(40, 64, 96, 80)
    for k in list(over):
        if hasattr(d, k):
            setattr(d, k, over.pop(k))
    at = {k: A + i * (1 << 20) for i, k in enumerate(["x", "w_gate", "w_up", "w_down", "h", "gate", "up", "y", "dy", "dx", "dw_gate", "dw_up", "dw_down", "ws"])}
    at.update(over)
    n = ctypes.c_size_t(0)
    size = jz.lib().jz_ffn_fwd_workspace_bytes if forward else jz.lib().jz_ffn_bwd_workspace_bytes
    size(ctypes.byref(d), ctypes.byref(n))
    names = ["x", "w_gate", "w_up", "w_down", "h", "gate", "up", "y", "ws"] if forward else ["x", "w_gate", "w_up", "w_down", "gate", "up", "h", "dy", "dx", "dw_gate",
                                                                                             "dw_up", "dw_down", "ws"]
    fn = jz.lib().jz_ffn_fwd if forward else jz.lib().jz_ffn_bwd
    return fn(ctypes.byref(d), *(at[k] for k in names), n.value if ws_bytes is None else ws_bytes, None)


@pytest.mark.parametrize("forward", [True, False])
def test_ffn_descriptors(jz, forward):
    for bad in (dict(rows=-1), dict(in_features=0), dict(hidden=-3), dict(out_features=0), dict(act=4), dict(act=-1), dict(dtype=3), dict(x_stride=63), dict(y_stride=-1),
                dict(dx_stride=5), dict(dy_stride=79)):
        assert ffn_call(jz, forward, **bad) == jz.JZ_ERR_SHAPE, bad
    for bad in (dict(dtype=2), dict(rows=(1 << 31) + 1), dict(hidden=(1 << 24) + 8), dict(x_stride=1 << 25)):
        assert ffn_call(jz, forward, **bad) == jz.JZ_ERR_UNSUPPORTED, bad
    n = ctypes.c_size_t(0)
    for fn in (jz.lib().jz_ffn_fwd_workspace_bytes, jz.lib().jz_ffn_bwd_workspace_bytes):
        assert fn(None, ctypes.byref(n)) == fn(ctypes.byref(jz.ffn_desc(1, 8, 8, 8)), None) == jz.JZ_ERR_NULL


def test_ffn_arguments(jz):
    for k in ("x", "w_gate", "w_up", "w_down", "h", "y", "gate", "up"):
        assert ffn_call(jz, True, **{k: None}) == jz.JZ_ERR_NULL, k        # of gate and up both or neither
    for k in ("x", "w_gate", "w_up", "w_down", "h", "y", "gate", "up"):
        assert ffn_call(jz, True, **{k: A + (40 << 20) + 8}) == jz.JZ_ERR_ALIGN, k
    for bad in (dict(h=A), dict(y=A + (4 << 20) + 64), dict(gate=A + (6 << 20)), dict(y=A + (3 << 20) + 16)):
        assert ffn_call(jz, True, **bad) == jz.JZ_ERR_ALIAS, bad
    assert ffn_call(jz, True, rows=0) == jz.JZ_OK
    for bad in (dict(x=None), dict(w_up=None), dict(gate=None), dict(up=None), dict(h=None), dict(dy=None), dict(dw_gate=None), dict(dw_up=None, dw_down=None),
                dict(dx=None, dw_gate=None, dw_up=None, dw_down=None)):
        assert ffn_call(jz, False, **bad) == jz.JZ_ERR_NULL, bad
    for k in ("x", "w_gate", "w_up", "w_down", "gate", "up", "h", "dy", "dx", "dw_gate", "dw_up", "dw_down", "ws"):
        assert ffn_call(jz, False, **{k: A + (40 << 20) + 8}) == jz.JZ_ERR_ALIGN, k
    for bad in (dict(dx=A + (8 << 20)), dict(dw_gate=A + (1 << 20) + 32), dict(dw_up=A + (12 << 20)), dict(ws=A + (9 << 20)), dict(dw_down=A + (13 << 20))):
        assert ffn_call(jz, False, **bad) == jz.JZ_ERR_ALIAS, bad
    assert ffn_call(jz, False, ws=None) == ffn_call(jz, False, ws_bytes=2 * 40 * 96 * 2 - 16) == jz.JZ_ERR_WORKSPACE


def test_ffn_workspace_without_rows(jz):
    """Without rows the backward call needs no workspace, but one that it is told of has to be there: odd feature counts are copied into it."""
    for k in (dict(ws=None), dict(ws=None, in_features=63)):
        assert ffn_call(jz, False, rows=0, ws_bytes=1 << 20, **k) == jz.JZ_ERR_WORKSPACE, k
    assert ffn_call(jz, False, rows=0, ws=A + (40 << 20) + 8, ws_bytes=1 << 20) == jz.JZ_ERR_ALIGN
    assert ffn_call(jz, True, rows=40, ws=None, ws_bytes=1 << 20) == jz.JZ_ERR_WORKSPACE
