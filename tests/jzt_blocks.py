"""Helpers of the residual-block operators' GPU tests: seeded tensors of the three element types and the per-element comparison."""
import numpy as np
import torch

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# one rounding to nearest, and half the spacing of the smallest numbers
ROUND = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
E32 = 2.0 ** -24


def randn(g, shape, dtype, std=1.0, mean=0.0):
    return torch.from_numpy(g.standard_normal(shape) * std + mean).to(dtype).to(DEV)


def wide(t):
    """float64 on the host."""
    return None if t is None else t.detach().cpu().double().numpy()


def nans(shape, dtype):
    """An output that nothing has been written to."""
    return torch.full(shape if isinstance(shape, tuple) else (shape,), float("nan"), dtype=dtype, device=DEV)


def check(got, ref, mag, c, what):
    """|got - ref| <= one rounding of the result + c roundings of FP32 of the size of the terms."""
    u, t = ROUND[got.dtype], TINY[got.dtype]
    g = wide(got)
    assert g.shape == ref.shape, what
    bound = u * np.abs(ref) + (1 + u) * c * E32 * mag + t
    over = np.abs(g - ref) - bound
    worst = np.unravel_index(np.argmax(np.where(np.isnan(over), np.inf, over)), over.shape) if over.size else None
    assert over.size == 0 or np.all(over <= 0), "%s: at %s got %r, exact %r, bound %r" % (what, worst, g[worst], ref[worst], bound[worst])
