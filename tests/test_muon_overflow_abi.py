"""Refusals of jz_muon_mp_overflow, found on the host before anything is launched (no GPU needed)."""
import ctypes
import math

from test_tokens_abi import A, STEP, jz, places, size, spread    # noqa: F401 (a fixture)


def overflow(jz, ws_bytes=None, hp=None, **over):
    d = jz.ortho_desc(2, 40, 60)
    spread(d, over)
    at = places(["state", "skip", "momentum", "grad", "flag", "ws"], over)
    n = size(jz, "jz_muon_mp_update_workspace_bytes", d)[1]
    return jz.lib().jz_muon_mp_overflow(ctypes.byref(d), ctypes.byref(jz.muon_hparams(**(hp or {}))), at["state"], at["skip"], at["momentum"], at["grad"], at["flag"], at["ws"],
                                        n if ws_bytes is None else ws_bytes, None)


def test_refusals(jz):    # noqa: F811
    assert overflow(jz, rows=0) == overflow(jz, out_dtype=1) == jz.JZ_ERR_SHAPE and overflow(jz, dtype=2, out_dtype=2) == overflow(jz, steps=100) == jz.JZ_ERR_UNSUPPORTED
    for bad in (dict(lr=math.nan), dict(momentum=math.inf), dict(weight_decay=math.nan), dict(update_scale=math.inf)):
        assert overflow(jz, hp=bad) == jz.JZ_ERR_SHAPE, bad
    for s in (0.0, -1.0, math.inf, math.nan):
        assert overflow(jz, hp=dict(loss_scale=s), state=None) == jz.JZ_ERR_SHAPE, s
    for k in ("momentum", "grad", "flag"):
        assert overflow(jz, **{k: None}) == jz.JZ_ERR_NULL, k
    n = size(jz, "jz_muon_mp_update_workspace_bytes", jz.ortho_desc(2, 40, 60))[1]
    assert overflow(jz, ws=None) == overflow(jz, ws_bytes=n - 1) == jz.JZ_ERR_WORKSPACE
    for k, by in (("state", 4), ("skip", 2), ("momentum", 8), ("grad", 8), ("flag", 2), ("ws", 8)):
        assert overflow(jz, **{k: A + 20 * STEP + by}) == jz.JZ_ERR_ALIGN, k
    names = ["state", "skip", "momentum", "grad", "flag", "ws"]
    reach = dict(state=8, skip=4, momentum=19200, grad=9600, flag=4, ws=n)
    for i, p in enumerate(names):
        for q in names[i + 1:]:
            if q in ("flag", "ws"):                                     # what is written
                assert overflow(jz, **{q: A + i * STEP}) == jz.JZ_ERR_ALIAS, (p, q)
                if reach[p] >= 32:
                    assert overflow(jz, **{q: A + i * STEP + (reach[p] - 1) // 16 * 16}) == jz.JZ_ERR_ALIAS, (p, q)
