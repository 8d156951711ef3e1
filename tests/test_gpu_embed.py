"""Embedding lookup and its table's gradient against their 64-bit definition: one rounding of the result, and one of FP32 for each term of a sum, the scale and what
was there (oracle.tokens.embed_bwd counts them).  Tokens that begin, end and go on at the edges of what a workgroup adds up, tokens outside the table, empty tables' rows."""
import numpy as np
import pytest
import torch

from jzt_blocks import DEV, TYPES, check, nans, randn, wide
from oracle import tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


def to_ids(a):
    return torch.from_numpy(np.asarray(a, np.int32)).to(DEV)


def run_bwd(jz, ids, dout, vocab, D, dtype, scale, before=None, out_stride=0, ws_extra=0):
    d = jz.embed_desc(len(ids), vocab, D, jz.dtype_of(dtype), jz.dtype_of(dout.dtype), scale, out_stride)
    ws = torch.full((jz.jz_embed_bwd_workspace_bytes(d) + ws_extra,), 0x5a, dtype=torch.uint8, device=DEV)
    out = nans((vocab, D), dtype) if before is None else before.clone()
    jz.jz_embed_bwd(d, to_ids(ids), dout, out, ws, accumulate=before is not None)
    torch.cuda.synchronize()
    return out


PAIRS = [("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 50, 64), (7, 3, 7), (300, 1000, 129), (64, 9, 4096), (1000, 5, 8), (5, 11, 2500), (2100, 700, 96)])
def test_both_ways(jz, types, T, V, D):
    g = np.random.default_rng([1, T, V, D])
    t, o = TYPES[types[0]], TYPES[types[1]]
    ids = g.integers(-1, V + 1, T)
    table, dout = randn(g, (V, D), t), randn(g, (T, D), o)
    scale = 1.7
    s32 = float(np.float32(scale))
    d = jz.embed_desc(T, V, D, jz.dtype_of(t), jz.dtype_of(o), scale)
    out = nans((T, D), o)
    jz.jz_embed_fwd(d, to_ids(ids), table, out)
    ref = tokens.embed_fwd(ids, wide(table), s32)
    check(out, ref, np.abs(ref), 1, "out")
    dt = run_bwd(jz, ids, dout, V, D, t, scale)
    ref, mag = tokens.embed_bwd(ids, wide(dout), V, s32)
    check(dt, ref, mag, 1, "dtable")
    before = randn(g, (V, D), t)
    dt = run_bwd(jz, ids, dout, V, D, t, scale, before)
    ref, mag = tokens.embed_bwd(ids, wide(dout), V, s32, wide(before))
    check(dt, ref, mag, 1, "dtable, added to")
    idle = np.ones(V, bool)
    idle[ids[(ids >= 0) & (ids < V)]] = False
    assert torch.equal(dt[torch.from_numpy(idle).to(DEV)], before[torch.from_numpy(idle).to(DEV)])


def runs(lengths, V, g):
    """Positions of tokens that occur so often, in an order that is no order."""
    ids = np.concatenate([np.full(n, v % V) for v, n in enumerate(lengths)])
    return g.permutation(ids)


@pytest.mark.parametrize("lengths", [[1000], [8, 8, 8, 8], [16, 16, 17], [15, 17, 33, 1, 2, 48, 49], [31, 1, 32, 64, 65, 7], [1, 40, 1, 40, 1, 300], [24, 0, 25, 23] * 6, [5000, 1, 3, 9000],
                                     [20000, 1, 1, 1, 30000, 63, 64, 65, 129], [0, 0, 1]])
@pytest.mark.parametrize("D", [24, 520])
def test_frequent_tokens(jz, lengths, D):
    """Pieces of 8, 16 and 32 positions (by their number), tokens of one to thousands of places across their borders."""
    g = np.random.default_rng([2, len(lengths), D])
    V = len(lengths) + 3
    ids = runs(lengths, V, g)
    dout = randn(g, (len(ids), D), torch.float32)
    dt = run_bwd(jz, ids, dout, V, D, torch.float32, 0.25)
    ref, mag = tokens.embed_bwd(ids, wide(dout), V, 0.25)
    check(dt, ref, mag, 1, "dtable")


@pytest.mark.parametrize("T", [1023, 1024, 1025, 4096, 4097, 16384, 16385, 20480, 100003])
@pytest.mark.parametrize("V", [1, 2, 511, 512, 70001, (1 << 18) - 1, (1 << 18)])
def test_every_place_goes_to_its_token(jz, T, V):
    """Whole numbers, whose sums are exact: one launch or several sort them, in one to three passes; the same bits each time."""
    g = np.random.default_rng([3, T, V])
    ids = np.minimum(V * g.random(T) ** 3, V - 1).astype(np.int64)
    ids[g.random(T) < 0.02] = -1
    ids[g.random(T) < 0.02] = V
    ids[0], ids[-1] = V - 1, 0
    dout = torch.from_numpy(g.integers(-8, 9, (T, 8))).to(DEV).float()
    ref, _ = tokens.embed_bwd(ids, wide(dout), V, 1.0)
    a = run_bwd(jz, ids, dout, V, 8, torch.float32, 1.0)
    assert np.array_equal(wide(a), ref)
    noise = randn(g, (T, 8), torch.float32)
    a, b = run_bwd(jz, ids, noise, V, 8, torch.float32, 1.0), run_bwd(jz, ids, noise, V, 8, torch.float32, 1.0, ws_extra=4096)
    assert torch.equal(a, b)


def test_the_largest_token_number(jz):
    V = (1 << 31) - 1
    d = jz.embed_desc(9, V, 1, jz.JZ_F16)
    ids = [V - 1, 0, -1, V - 1, -(1 << 31), 5, V - 2, 0, V - 1]
    table = torch.zeros(V, dtype=torch.float16, device=DEV)
    table[0], table[5], table[V - 2], table[V - 1] = 1, 2, 3, 4
    out = nans((9, 1), torch.float16)
    jz.jz_embed_fwd(d, to_ids(ids), table, out)
    assert out.view(-1).tolist() == [4, 1, 0, 4, 0, 2, 3, 1, 4]
    ws = torch.empty(jz.jz_embed_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    jz.jz_embed_bwd(d, to_ids(ids), out, table, ws)
    torch.cuda.synchronize()
    assert [float(table[i]) for i in (0, 1, 5, V - 2, V - 1)] == [2, 0, 2, 3, 12] and float(table.float().sum()) == 19


def test_offsets_beyond_32_bits(jz):
    """A table of 4.4 billion elements and a stream whose rows lie far apart."""
    V, D, T, ld = 1100000, 4000, 40, 1 << 24
    table = torch.zeros((V, D), dtype=torch.float16, device=DEV)
    ids = [V - 1 - 27 * i for i in range(T)]
    for i, v in enumerate(ids):
        table[v] = i + 1
    room = torch.full((T * ld,), 7.0, dtype=torch.float32, device=DEV)
    out = room.as_strided((T, D), (ld, 1))
    d = jz.embed_desc(T, V, D, jz.JZ_F16, jz.JZ_F32, 2.0, ld)
    jz.jz_embed_fwd(d, to_ids(ids), table, out)
    want = (torch.arange(T, device=DEV).float() + 1) * 2
    assert torch.equal(out, want[:, None].expand(T, D)) and bool((room[D:ld] == 7).all()) and bool((room[(T - 1) * ld + D:] == 7).all())
    ws = torch.empty(jz.jz_embed_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    table.fill_(float("nan"))
    jz.jz_embed_bwd(d, to_ids(ids), out, table, ws)
    torch.cuda.synchronize()
    assert torch.equal(table[torch.tensor(ids, device=DEV)], (2 * want).half()[:, None].expand(T, D))
    assert float(table.sum(dtype=torch.float64)) == 2 * D * float(want.sum())


def test_masked_places_are_not_read(jz):
    g = np.random.default_rng(5)
    ids = np.array([3, -1, 0, 9, 3, 10, 0])
    dout = randn(g, (7, 40), torch.float32)
    dout[[1, 5]] = float("nan")
    dt = run_bwd(jz, ids, dout, 10, 40, torch.float32, 1.0)
    ref, mag = tokens.embed_bwd(ids, np.where(np.isnan(wide(dout)), 0, wide(dout)), 10, 1.0)
    check(dt, ref, mag, 1, "dtable")
    table = randn(g, (10, 40), torch.float16)
    table[4] = float("nan")                         # no token asks for it
    out = nans((7, 40), torch.float16)
    jz.jz_embed_fwd(jz.embed_desc(7, 10, 40), to_ids(ids), table, out)
    assert bool((out[[1, 5]] == 0).all()) and bool(torch.isfinite(out).all())
    none = run_bwd(jz, np.full(300, -1), nans((300, 16), torch.float32), 6, 16, torch.float16, 1.0)
    assert bool((none == 0).all())


def test_rows_between_and_behind_are_left_alone(jz):
    g = np.random.default_rng(6)
    T, V, D, ld = 33, 20, 100, 160
    ids = g.integers(0, V, T)
    table = randn(g, (V, D), torch.bfloat16)
    room = torch.full(((T + 4) * ld,), 5.0, dtype=torch.bfloat16, device=DEV)
    out = room[:T * ld].view(T, ld)[:, :D]
    jz.jz_embed_fwd(jz.embed_desc(T, V, D, jz.JZ_BF16, None, 1.0, ld), to_ids(ids), table, out)
    assert torch.equal(out, table[torch.from_numpy(ids).to(DEV)])
    assert bool((room[:T * ld].view(T, ld)[:, D:] == 5).all()) and bool((room[T * ld:] == 5).all())


def test_without_tokens(jz):
    d = jz.embed_desc(0, 7, 12)
    none = torch.empty((0, 12), dtype=torch.float16, device=DEV)
    jz.jz_embed_fwd(d, to_ids([]), torch.ones((7, 12), dtype=torch.float16, device=DEV), none)
    out = nans((7, 12), torch.float16)
    ws = torch.empty(jz.jz_embed_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    jz.jz_embed_bwd(d, to_ids([]), none, out, ws, accumulate=True)
    assert bool(torch.isnan(out).all())
    jz.jz_embed_bwd(d, to_ids([]), none, out, ws)
    assert bool((out == 0).all())


def test_the_gradient_against_differences(jz):
    g = np.random.default_rng(7)
    T, V, D = 50, 12, 16
    ids = g.integers(0, V, T)
    table, c = randn(g, (V, D), torch.float32), randn(g, (T, D), torch.float32)
    d = jz.embed_desc(T, V, D, jz.JZ_F32, None, 3.0)

    def value(t):
        out = nans((T, D), torch.float32)
        jz.jz_embed_fwd(d, to_ids(ids), t, out)
        return float((out.double() * c.double()).sum())
    grad = run_bwd(jz, ids, c, V, D, torch.float32, 3.0)
    step = 2.0 ** -4
    for v, k in ((0, 0), (5, 15), (11, 7)):
        up, down = table.clone(), table.clone()
        up[v, k] += step
        down[v, k] -= step
        n = int((ids == v).sum())
        # the lookups and their difference are off by a rounding of FP32 each: 3 * 4 * 2^-24 a term at most
        assert abs((value(up) - value(down)) / (2 * step) - float(grad[v, k])) <= (n + 2) * 2.0 ** -24 * 12 * 4 / step


@pytest.mark.parametrize("T", [900, 20000])
def test_in_a_graph_and_on_another_stream(jz, T):
    g = np.random.default_rng(8)
    V, D = 3000, 72
    ids, dout = to_ids(np.minimum(g.exponential(200, T), V - 1)), randn(g, (T, D), torch.float16)
    d = jz.embed_desc(T, V, D)
    ws = torch.empty(jz.jz_embed_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    out, again = nans((V, D), torch.float16), nans((V, D), torch.float16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    jz.jz_embed_bwd(d, ids, dout, out, ws, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jz.jz_embed_bwd(d, ids, dout, again, ws)
    for k in range(4):
        if k:                                       # other tokens, by the same graph
            ids.copy_(to_ids(g.integers(-1, V, T)))
            jz.jz_embed_bwd(d, ids, dout, out, ws)
        again.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, again), k


@pytest.mark.parametrize("types,T,D", [(("bf16", "bf16"), 16500, 4097), (("f16", "f32"), 16500, 2050), (("f32", "f32"), 8200, 4100), (("bf16", "f32"), 40000, 1003), (("f16", "f16"), 33000, 2048)])
def test_lookups_past_the_caches(jz, types, T, D):
    """Results of 128 MiB and more; half of a number is exact."""
    V, dt, out = 3001, TYPES[types[0]], TYPES[types[1]]
    g = torch.Generator(DEV).manual_seed(T)
    table = torch.randint(-100, 101, (V, D), generator=g, device=DEV).to(dt)
    ids = torch.randint(-2, V + 2, (T,), generator=g, device=DEV, dtype=torch.int32)
    y = torch.full((T, D), 7.0, dtype=out, device=DEV)
    jz.jz_embed_fwd(jz.embed_desc(T, V, D, jz.dtype_of(dt), jz.dtype_of(out), 0.5), ids, table, y)
    there = (ids >= 0) & (ids < V)
    assert torch.equal(y, torch.where(there[:, None], table[ids.clamp(0, V - 1).long()].to(out) * 0.5, torch.zeros((), dtype=out, device=DEV)))


@pytest.mark.parametrize("types,T,V,D", [(("f16", "f32"), 33000, 70001, 1024), (("bf16", "bf16"), 34000, 17000, 4096), (("f16", "f32"), 18000, 20000, 4096), (("bf16", "f32"), 5000, 70001, 1001),
                                         (("f32", "f32"), 70000, 40000, 512), (("f16", "f16"), 35000, 300, 2049), (("f16", "f16"), 33600, 400, 2048)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradients_past_the_caches(jz, types, T, V, D, accumulate):
    """Tables and rows of 128 MiB and more; sums of whole numbers are exact."""
    dt, out = TYPES[types[0]], TYPES[types[1]]
    g = torch.Generator(DEV).manual_seed(T + V)
    ids = torch.where(torch.rand(T, generator=g, device=DEV) < 0.01, torch.full((), V // 2, device=DEV), torch.randint(-2, V + 2, (T,), generator=g, device=DEV)).int()
    dout = torch.randint(-1, 2, (T, D), generator=g, device=DEV).to(out)
    before = torch.randint(-1, 2, (V, D), generator=g, device=DEV).to(dt) if accumulate else torch.full((V, D), float("nan"), dtype=dt, device=DEV)
    got, d = before.clone(), jz.embed_desc(T, V, D, jz.dtype_of(dt), jz.dtype_of(out), 2.0)
    jz.jz_embed_bwd(d, ids, dout, got, torch.full((jz.jz_embed_bwd_workspace_bytes(d),), 0x33, dtype=torch.uint8, device=DEV), accumulate=accumulate)
    there = (ids >= 0) & (ids < V)
    want = torch.zeros((V, D), device=DEV).index_add_(0, ids[there].long(), dout[there].float()) * 2
    assert float(want.abs().max()) <= 250       # with one more, whole numbers in eight bits
    assert torch.equal(got.float(), want + before.float() if accumulate else want)
