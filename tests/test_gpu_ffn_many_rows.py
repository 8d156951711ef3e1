"""The feed-forward block of 2^31 rows, more than one launch's worth of tiles and of copies, one feature each, so that the formulas are elementwise: checked piece by
piece in FP32, stage by stage on what the calls leave.

u = 2^-11.  h is one rounding of FP32's result (2^-18 for exp, reciprocal and products); y = h / 2 exactly.  dx: dgate and dup carry a rounding each, and the result one.
Weight gradients: sums of 2^31 terms of either sign, each with at most three roundings of u / sqrt(3), independent: 2^-11 of the root of the sum of their squares; FP32 sums of 2^26
terms in a split, sixteen at a time, keep about 2^-24 sqrt(2^22) = 2^-13 of it: 2^-7 is asked for (a launch of the last 2^-8 of the rows left out would be 2^-4), and the store's u."""
import pytest
import torch

pytestmark = pytest.mark.gpu
M, PIECE = 1 << 31, 1 << 27
G, U, D = 1.25, -0.75, 0.5


def randn(std, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.empty(M, 1, dtype=torch.float16, device="cuda")
    for at in range(0, M, PIECE):
        t[at:at + PIECE] = torch.randn(PIECE, 1, generator=g, device="cuda") * std
    return t


def empty():
    return torch.full((M, 1), float("nan"), dtype=torch.float16, device="cuda")


def weight(v):
    return torch.full((1, 1), v, dtype=torch.float16, device="cuda")


def workspace(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda") if n else None


@pytest.fixture
def memory():
    torch.cuda.empty_cache()
    yield torch.cuda.mem_get_info()[0]
    torch.cuda.empty_cache()


@pytest.mark.parametrize("copies", [False, True])
def test_forward(memory, copies):
    from paper_1807_11205_amd import api
    if memory < 100 << 30:
        pytest.skip("less than 100 GiB of free GPU memory")
    d = api.ffn_desc(M, 1, 1, 1)
    x, h, y, ws = randn(1.0, 1), empty(), empty(), workspace(api.jz_ffn_fwd_workspace_bytes(d) if copies else 0)
    api.jz_ffn_fwd(d, x, weight(G), weight(U), weight(D), h, y, ws=ws)
    for at in range(0, M, PIECE):
        v = x[at:at + PIECE].float()
        want = v * G * torch.sigmoid(v * G) * (v * U)
        assert torch.all((h[at:at + PIECE].float() - want).abs() <= (2.0 ** -11 + 2.0 ** -18) * want.abs() + 2.0 ** -25), at
        assert torch.equal(y[at:at + PIECE], h[at:at + PIECE] * D), at


def test_backward(memory):
    from paper_1807_11205_amd import api
    if memory < 220 << 30:
        pytest.skip("less than 220 GiB of free GPU memory")
    d = api.ffn_desc(M, 1, 1, 1)
    x, gate, up, h, dy, dx = randn(1.0, 1), randn(1.0, 2), randn(1.0, 3), randn(1.0, 4), randn(0.05, 5), empty()
    dws = [weight(float("nan")) for _ in range(3)]
    ws = workspace(api.jz_ffn_bwd_workspace_bytes(d))
    api.jz_ffn_bwd(d, x, weight(G), weight(U), weight(D), gate, up, h, dy, dx, *dws, ws=ws)
    total, squares = [0.0] * 3, [0.0] * 3
    for at in range(0, M, PIECE):
        s = slice(at, at + PIECE)
        v = dy[s].float() * D
        g = gate[s].float()
        a = torch.sigmoid(g)
        du, dg = v * g * a, v * up[s].float() * (a * (1 + g * (1 - a)))
        want = dg * G + du * U
        # the slope is a difference of terms of up to 1 + |gate|: FP32's roundings of those
        bound = 2.0 ** -11 * (want.abs() + 1.1 * (dg.abs() * G + du.abs() * -U)) + 2.0 ** -18 * v.abs() * (1 + g.abs()) * (1 + up[s].float().abs()) + 2.0 ** -23
        assert torch.all((dx[s].float() - want).abs() <= bound), at
        for i, t in enumerate((dg * x[s], du * x[s], dy[s].float() * h[s])):
            total[i] += t.double().sum().item()
            squares[i] += t.double().square().sum().item()
    for i in range(3):
        got = float(dws[i])
        assert abs(got - total[i]) <= 2.0 ** -7 * squares[i] ** 0.5 + 2.0 ** -11 * abs(total[i]), (i, got, total[i], squares[i] ** 0.5)
