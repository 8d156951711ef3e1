"""Grids of the residual-block operators over the whole range of what their descriptors accept (no GPU: launches are recorded by a library in front of the HIP
runtime, in a process of its own).  A launch has fewer than 2^32 lanes along x and at most 65535 workgroups along y, else the runtime refuses it."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
A = 1 << 58             # tensors' addresses, far apart; never followed


class Recorded:
    """In the child process: the library behind the recorder."""

    def __init__(self, recorder):
        self.rec = ctypes.CDLL(recorder, mode=ctypes.RTLD_GLOBAL)
        self.lib = ctypes.CDLL(os.path.join(ROOT, "paper_1807_11205_amd", "libjz.so"))

    def call(self, name, *args):
        self.rec.forget()
        conv = [a if not isinstance(a, int) or isinstance(a, bool) else ctypes.c_void_p(a) for a in args]
        status = getattr(self.lib, name)(*conv)
        out = (ctypes.c_uint * 6)()
        grids = []
        for i in range(min(self.rec.launches(), 4096)):
            self.rec.launch(i, out)
            grids.append(list(out))
        return dict(status=status, launches=self.rec.launches(), grids=grids)


def tensors(n):
    return [A * (i + 1) for i in range(n)]


def norm_desc(rows, channels, dtype=0):
    class D(ctypes.Structure):
        _fields_ = [("rows", ctypes.c_int64), ("channels", ctypes.c_int), ("rows_per_group", ctypes.c_int64), ("dtype", ctypes.c_int), ("res_dtype", ctypes.c_int),
                    ("eps", ctypes.c_float), ("res_scale", ctypes.c_float), ("branch_scale", ctypes.c_float)]
    return D(rows, channels, 0, dtype, dtype, 1e-5, 1.0, 1.0)


def child(recorder, job):
    r = Recorded(recorder)
    print(json.dumps([JOBS[job["job"]](r, *c) for c in job["cases"]]))


def norm_forward(r, rows, channels):
    d = norm_desc(rows, channels)
    return r.call("jz_norm_residual_fwd", ctypes.byref(d), *tensors(9), None)


def norm_backward(r, rows, channels):
    d, n = norm_desc(rows, channels), ctypes.c_size_t(0)
    r.lib.jz_norm_residual_bwd_workspace_bytes(ctypes.byref(d), ctypes.byref(n))
    return r.call("jz_norm_residual_bwd", ctypes.byref(d), *tensors(15), ctypes.c_size_t(n.value), None)


def ffn_desc(rows, D, F, O):
    class D_(ctypes.Structure):
        _fields_ = [("rows", ctypes.c_int64), ("in_features", ctypes.c_int), ("hidden", ctypes.c_int), ("out_features", ctypes.c_int), ("act", ctypes.c_int),
                    ("dtype", ctypes.c_int), ("x_stride", ctypes.c_int64), ("y_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64)]
    return D_(rows, D, F, O, 0, 0, 0, 0, 0, 0)


def ffn_forward(r, rows, D, F, O, all_of_it):
    d, n = ffn_desc(rows, D, F, O), ctypes.c_size_t(0)
    status = r.lib.jz_ffn_fwd_workspace_bytes(ctypes.byref(d), ctypes.byref(n))
    if not all_of_it:
        n.value = 0
    got = r.call("jz_ffn_fwd", ctypes.byref(d), *tensors(9), n, None)
    return dict(got, asked=status)


def ffn_backward(r, rows, D, F, O, all_of_it):
    d, n = ffn_desc(rows, D, F, O), ctypes.c_size_t(0)
    status = r.lib.jz_ffn_bwd_workspace_bytes(ctypes.byref(d), ctypes.byref(n))
    if not all_of_it:
        n.value = 2 * ((rows * ((F + 7) // 8 * 8) * 2 + 255) // 256 * 256)
    got = r.call("jz_ffn_bwd", ctypes.byref(d), *tensors(13), n, None)
    return dict(got, asked=status)


JOBS = dict(ffn_forward=ffn_forward, ffn_backward=ffn_backward, norm_forward=norm_forward, norm_backward=norm_backward)


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    from paper_1807_11205_amd import api
    if not os.path.exists(api.LIB_PATH):
        from paper_1807_11205_amd import build
        build.build()
    out = tmp_path_factory.mktemp("recorder") / "librecorder.so"
    subprocess.run([os.environ.get("CC", "gcc"), "-O1", "-shared", "-fPIC", "-o", str(out), os.path.join(HERE, "launch_recorder.c")], check=True)
    return str(out)


def run(recorder, job, cases):
    r = subprocess.run([sys.executable, os.path.abspath(__file__), recorder, json.dumps(dict(job=job, cases=cases))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    return list(zip(cases, json.loads(r.stdout.splitlines()[-1])))


def fits(g):
    return all(v > 0 for v in g) and g[0] * g[3] < 1 << 32 and g[1] <= 65535 and g[2] <= 65535


ROWS = [1, 5, 1 << 20, (1 << 24) - 1, 1 << 24, (1 << 24) + 1, (1 << 26) - 4, 1 << 26, (1 << 26) + 3, (1 << 30) + 7, (1 << 31) - 256]


def test_norms_forward(recorder):
    for (rows, channels), got in run(recorder, "norm_forward", [(m, c) for m in ROWS for c in (1, 8, 64, 512, 1000, 1024, 1025, 4096, 8192, 16384)]):
        assert got["status"] == 0 and got["launches"] >= 1, (rows, channels, got)
        assert all(fits(g) for g in got["grids"]), (rows, channels, got)
        each = 4 if channels <= 1024 else 1
        assert sum(g[0] for g in got["grids"]) == -(-rows // each), (rows, channels, got)


def test_norms_backward(recorder):
    for (rows, channels), got in run(recorder, "norm_backward", [(m, c) for m in ROWS for c in (1, 8, 64, 512, 1000, 1024, 1025, 4096, 8192, 16384)]):
        assert got["status"] == 0 and got["launches"] == 2, (rows, channels, got)
        assert all(fits(g) for g in got["grids"]), (rows, channels, got)


# rows and features whose tensors have up to 2^38 elements each
BLOCKS = [(m, d, f, o) for m in (1, 64, 65, 1 << 20, (1 << 30) + 1, (1 << 31) - 1, 1 << 31)
          for d, f, o in ((1, 1, 1), (8, 8, 8), (9, 8, 1), (64, 64, 64), (64, 65, 64), (127, 128, 120), (1000, 2730, 1000), (1 << 14, 1 << 14, 1 << 14), (1 << 24, 8, 8),
                          (8, 1 << 24, 8), (1, (1 << 24) - 1, 1), (1, 1, 1 << 24), ((1 << 24) - 3, 9, 1 << 24))
          if m * max(d, f, o) <= 1 << 38]


@pytest.mark.parametrize("job", ["ffn_forward", "ffn_backward"])
@pytest.mark.parametrize("all_of_it", [True, False])
def test_feed_forward_block(recorder, job, all_of_it):
    for (m, d, f, o, _), got in run(recorder, job, [(*b, all_of_it) for b in BLOCKS]):
        assert got["status"] == got["asked"] == 0 and got["launches"] >= 2, (m, d, f, o, got)
        assert all(fits(g) for g in got["grids"]), (m, d, f, o, got)
        if m > 64:              # every product of the rows' has a workgroup for each of its tiles, which are 256 x 256 at most
            cols = (2 * ((f + 31) // 32 * 32), o) if job == "ffn_forward" else (f, d)
            assert sum(g[0] * g[1] for g in got["grids"]) >= sum(-(-m // 256) * -(-c // 256) for c in cols), (m, d, f, o, got)


# (product, tile, are sums shared) by sizes; test_gpu_block_variants.py compares the results of these
PLANS = [((7536, 8, 1928, 648), "dh", 256, False), ((7048, 56, 2464, 2552), "dh", 256, True), ((136, 8, 8, 696), "dh", 128, True), ((2240, 2120, 3664, 16), "glu", 256, True),
         ((968, 120, 7032, 4192), "down", 256, True), ((8136, 136, 5944, 152), "dw", 256, True), ((8272, 416, 3640, 40), "dx", 256, True), ((136, 672, 8, 8), "glu", 128, True),
         ((80, 8, 696, 8), "down", 128, True), ((672, 8, 8, 8), "dw", 128, True), ((152, 8, 360, 8), "dx", 128, True)]


def readings(grids, products):
    """What the launches of a call may be: a product's tiles (512 or 256 lanes) each, and one that joins, which has tile^2 / 8 / 256 workgroups along x (half as many
    for gate and up)."""
    if not products:
        return [] if grids else [{}]
    if not grids:
        return []
    tile = 256 if grids[0][3] == 512 else 128
    res = [{products[0]: (tile, False), **r} for r in readings(grids[1:], products[1:])]
    if len(grids) > 1 and grids[1][0] == tile * tile // (4096 if products[0] == "glu" else 2048) and grids[1][3] == 256:
        res += [{products[0]: (tile, True), **r} for r in readings(grids[2:], products[1:])]
    return res


def test_sizes_that_stand_for_a_plan_have_it(recorder):
    got = {job: dict((tuple(c[:4]), g["grids"]) for c, g in run(recorder, job, [(*p[0], True) for p in PLANS])) for job in ("ffn_forward", "ffn_backward")}
    for size, product, tile, shared in PLANS:
        forward = product in ("glu", "down")
        found = {r[product] for r in readings(got["ffn_forward" if forward else "ffn_backward"][size], ["glu", "down"] if forward else ["dh", "dx", "dw"])}
        assert (tile, shared) in found and (tile == 128 or len(found) == 1), (size, product, found)


def test_blocks_larger_than_any_memory_are_refused(recorder):
    sizes = [(1 << 31, 129, 8, 8), (1 << 31, 8, 129, 8), (1 << 31, 8, 8, 129), (1, 1 << 24, (1 << 14) + 1, 8), (1, 8, 1 << 24, (1 << 14) + 1), (1 << 31, 1 << 24, 1 << 24, 1 << 24)]
    for job in ("ffn_forward", "ffn_backward"):
        for c, got in run(recorder, job, [(*z, False) for z in sizes]):
            assert got["status"] == got["asked"] == -3 and got["launches"] == 0, (c, got)


if __name__ == "__main__":
    child(sys.argv[1], json.loads(sys.argv[2]))
