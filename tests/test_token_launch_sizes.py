"""Grids of the embedding, orthogonalisation and 8-bit entry points over the whole range of what their descriptors accept (no GPU: launches are recorded, see
test_launch_sizes.py).  A launch has fewer than 2^32 lanes along x and at most 65535 workgroups along y."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, HERE)
from test_launch_sizes import Recorded, fits, recorder, tensors  # noqa: E402,F401

i64, ci, cf = ctypes.c_int64, ctypes.c_int, ctypes.c_float


class EmbedDesc(ctypes.Structure):
    _fields_ = [("tokens", i64), ("vocab", ci), ("channels", ci), ("dtype", ci), ("out_dtype", ci), ("scale", cf), ("out_stride", i64)]


class OrthoDesc(ctypes.Structure):
    _fields_ = [("count", i64), ("rows", ci), ("cols", ci), ("stride", i64), ("dtype", ci), ("out_dtype", ci), ("steps", ci), ("a", cf), ("b", cf), ("c", cf), ("eps", cf)]


class LinearDesc(ctypes.Structure):
    _fields_ = [("rows", i64), ("in_features", ci), ("out_features", ci), ("dtype", ci), ("x_stride", i64), ("y_stride", i64)]


class FfnDesc(ctypes.Structure):
    _fields_ = [("rows", i64), ("in_features", ci), ("hidden", ci), ("out_features", ci), ("act", ci), ("dtype", ci), ("x_stride", i64), ("y_stride", i64), ("dx_stride", i64),
                ("dy_stride", i64)]


class Hparams(ctypes.Structure):
    _fields_ = [("lr", cf), ("momentum", cf), ("weight_decay", cf), ("update_scale", cf), ("loss_scale", cf), ("nesterov", ci)]


def room(r, name, d):
    n = ctypes.c_size_t(0)
    return getattr(r.lib, name)(ctypes.byref(d), ctypes.byref(n)), n


def embed_forward(r, tokens, vocab, channels):
    d = EmbedDesc(tokens, vocab, channels, 0, 0, 1.0, 0)
    return r.call("jz_embed_fwd", ctypes.byref(d), *tensors(3), None)


def embed_backward(r, tokens, vocab, channels):
    d = EmbedDesc(tokens, vocab, channels, 0, 0, 1.0, 0)
    asked, n = room(r, "jz_embed_bwd_workspace_bytes", d)
    t = tensors(4)
    return dict(r.call("jz_embed_bwd", ctypes.byref(d), t[0], t[1], ctypes.c_int(0), t[2], t[3], n, None), asked=asked)


def ortho_desc(count, rows, cols, dtype):
    return OrthoDesc(count, rows, cols, 0, dtype, dtype, 5, 3.4445, -4.775, 2.0315, 1e-7)


def ortho(r, count, rows, cols):
    d = ortho_desc(count, rows, cols, 2)
    asked, n = room(r, "jz_orthogonalize_workspace_bytes", d)
    return dict(r.call("jz_orthogonalize", ctypes.byref(d), *tensors(3), n, None), asked=asked)


def muon(r, count, rows, cols):
    d, hp = ortho_desc(count, rows, cols, 0), Hparams(0.1, 0.9, 0.0, 1.0, 1.0, 1)
    asked, n = room(r, "jz_muon_mp_update_workspace_bytes", d)
    return dict(r.call("jz_muon_mp_update", ctypes.byref(d), ctypes.byref(hp), None, None, *tensors(6), n, None), asked=asked)


def linear(r, M, K, N):
    d = LinearDesc(M, K, N, 0, 0, 0)
    asked, n = room(r, "jz_linear_i8_workspace_bytes", d)
    return dict(r.call("jz_linear_i8", ctypes.byref(d), *tensors(5), n, None), asked=asked)


def block(r, M, D, F, O):
    d = FfnDesc(M, D, F, O, 0, 0, 0, 0, 0, 0)
    asked, n = room(r, "jz_ffn_i8_workspace_bytes", d)
    return dict(r.call("jz_ffn_i8_fwd", ctypes.byref(d), *tensors(9), n, None), asked=asked)


JOBS = dict(embed_forward=embed_forward, embed_backward=embed_backward, ortho=ortho, muon=muon, linear=linear, block=block)


def run(recorder, job, cases):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, json.dumps(dict(job=job, cases=cases))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return list(zip(cases, json.loads(r.stdout.splitlines()[-1])))


TABLES = [(t, v, c) for t in (1, 1024, 1025, 16384, 16385, 1 << 24, (1 << 31) - 1) for v, c in ((1, 1), (50000, 64), ((1 << 31) - 1, 128), (1 << 14, 1 << 24), (7, 129), (1 << 18, 1 << 20))
          if t * c <= 1 << 38 and v * c <= 1 << 38]


@pytest.mark.parametrize("job", ["embed_forward", "embed_backward"])
def test_embedding(recorder, job):  # noqa: F811
    for (t, v, c), got in run(recorder, job, TABLES):
        assert got["status"] == 0 and got["launches"] >= 1, (t, v, c, got)
        assert all(fits(g) for g in got["grids"]), (t, v, c, got)


MATRICES = [(1, 1, 1), (1, 1 << 17, 1), (65535, 1, 1), (65535, 300, 700), (65535, 724, 700), (1, 1 << 17, 1 << 17), (2, 1 << 17, 1 << 17), (1, 128, 1 << 17), (2047, 128, 1 << 17), (65535, 128, 128),
            (65535, 129, 129), (1000, 2048, 5632), (1 << 11, 4096, 4096)]


@pytest.mark.parametrize("job", ["ortho", "muon"])
def test_orthogonalisation(recorder, job):  # noqa: F811
    for (b, r, c), got in run(recorder, job, MATRICES):
        assert got["status"] == got["asked"] == 0 and got["launches"] >= 8, (b, r, c, got)
        assert all(fits(g) for g in got["grids"]), (b, r, c, got)


LAYERS = [(m, k, n) for m in (1, 4, 5, 64, 65, 1 << 20, (1 << 30) + 1, 1 << 31) for k, n in ((1, 1), (16, 128), (131072, 8), (131072, 1 << 21), (64, 1 << 24), (1000, 2731))
          if m * max(k, n) <= 1 << 38]


def test_linear(recorder):  # noqa: F811
    for (m, k, n), got in run(recorder, "linear", LAYERS):
        assert got["status"] == got["asked"] == 0 and got["launches"] >= 1, (m, k, n, got)
        assert all(fits(g) for g in got["grids"]), (m, k, n, got)
        if m > 64:              # a workgroup for each tile, which is 256 x 256 at most
            assert sum(g[0] for g in got["grids"][1:]) >= -(-m // 256) * -(-n // 256), (m, k, n, got)
        else:
            assert got["grids"][-1][0] == -(-n // 16), (m, k, n, got)


def test_block(recorder):  # noqa: F811
    cases = [(m, d, f, o) for m in (1, 4, 5, 64, 65, 1 << 20, 1 << 31) for d, f, o in ((1, 1, 1), (16, 128, 64), (131072, 131072, 8), (1, 131072, 1 << 21)) if m * max(d, f, o) <= 1 << 38]
    for (m, d, f, o), got in run(recorder, "block", cases):
        assert got["status"] == got["asked"] == 0 and got["launches"] >= 2, (m, d, f, o, got)
        assert all(fits(g) for g in got["grids"]), (m, d, f, o, got)


if __name__ == "__main__":
    r = Recorded(sys.argv[1])
    job = json.loads(sys.argv[2])
    print(json.dumps([JOBS[job["job"]](r, *c) for c in job["cases"]]))
