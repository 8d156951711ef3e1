"""The norms of more rows than one launch takes (2^26 of up to 1024 channels), against the formula in FP32 piece by piece: FP16 results, so within one rounding
and a few of FP32's (2^-11 + 2^-18, relative; numbers of the size of one, so nothing is lost below FP16's smallest)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_behind_the_first_launch(in_place):
    from paper_1807_11205_amd import api
    C, per, groups = 8, 64, (1 << 20) + 1
    rows, eps, h, f = groups * per, 1e-5, torch.float16, torch.float32
    g = torch.Generator(device="cuda").manual_seed(3)
    r, y = (torch.randn(rows, C, generator=g, device="cuda", dtype=h) for _ in range(2))
    gate, w_post, w_pre = torch.randn(groups, C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    keep = r.clone()
    r_out = r if in_place else torch.full_like(r, float("nan"))
    n, k1, k2 = torch.full_like(r, float("nan")), torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    d = api.norm_residual_desc(rows, C, per, api.JZ_F16, api.JZ_F16, eps, 1.0, 0.5)
    api.jz_norm_residual_fwd(d, r, y, w_post, gate, w_pre, r_out, n, k1, k2)
    u = 2.0 ** -11 + 2.0 ** -18
    for at in range(0, rows, 1 << 23):
        s = slice(at, min(at + (1 << 23), rows))
        yy = y[s].to(f)
        a = 1 / torch.sqrt((yy * yy).mean(1) + eps)
        p = 0.5 * gate[at // per:(s.stop + per - 1) // per].repeat_interleave(per, 0) * (yy * a[:, None] * w_post)
        out = keep[s].to(f) + p
        b = 1 / torch.sqrt((out * out).mean(1) + eps)
        assert torch.all((k1[s] - a).abs() <= 2.0 ** -18 * a), at
        # out is a difference where its terms have opposite signs: FP32 roundings of the terms
        size = keep[s].to(f).abs() + p.abs()
        assert torch.all((r_out[s].to(f) - out).abs() <= u * out.abs() + 2.0 ** -18 * size + 2.0 ** -25), at
        # through the second norm, with the relative error of its own sum of squares
        change = b ** 3 * (out.abs() * size).mean(1)
        assert torch.all((k2[s] - b).abs() <= 2.0 ** -18 * torch.maximum(b, change)), at
        want = out * b[:, None] * w_pre
        assert torch.all((n[s].to(f) - want).abs() <= u * want.abs() + 2.0 ** -17 * (size * torch.maximum(b, change)[:, None] * w_pre.abs()) + 2.0 ** -25), at
