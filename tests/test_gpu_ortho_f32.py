"""FP32 results of the orthogonalisation against 64 bits, beside the same formulas in FP32.

How much further off they may be than those.  Rounded to 24 bits, an element of a binade 2^e is off by 2^-23 2^e / sqrt(12) = 2^(e - 24.8) in the root mean square.  As two FP16 parts: what the high one
leaves is spread over 2^-10 2^e, its root mean square 2^-10 2^e / sqrt(12), and rounding that to 11 bits leaves 2^-12.3 of it (a step / sqrt(12) over a mean of 1.4 steps' worth of numbers):
2^(e - 24.1), 1.6 times as much.  A product has two such operands and leaves out low x low, (2^-10 / sqrt(12))^2 of two numbers of 1.4, 2^-24.3 or 1.4 times FP32's rounding: altogether
sqrt(2 * 1.6^2 + 1.4^2) / sqrt(2) = 1.9 times, and less by as much as the FP32 sums add that both have.  Over a thousand elements and more these root mean squares scatter, and the errors of the steps do not
all grow alike: a third more.  (What the iteration makes of its errors is the same in both where both take the same steps.)"""
import numpy as np
import pytest
import torch

from jzt_blocks import DEV, wide
from oracle import tokens
from test_gpu_ortho import C32, EPS, jz, run    # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu
FACTOR = 2.5


def in_fp32(x):
    x = x / (x.double().norm() + EPS).float()
    tall = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if tall else x
    for _ in range(5):
        A = x @ x.T
        x = C32[0] * x + (C32[1] * A + C32[2] * (A @ A)) @ x
    return x.T if tall else x


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
@pytest.mark.parametrize("B,R,C", [(64, 16, 16), (32, 40, 32), (16, 64, 64), (8, 128, 128), (4, 300, 120), (2, 128, 512), (1, 64, 3000), (2, 200, 200), (2, 200, 420), (1, 512, 800), (1, 1024, 2816)])
def test_beside_fp32(jz, B, R, C, dtype):    # noqa: F811
    g = np.random.default_rng([3, B, R, C])
    x = torch.from_numpy(g.standard_normal((B, R, C))).to(dtype)
    y, own, plain, size = wide(run(jz, x.to(DEV), torch.float32)), 0.0, 0.0, 0.0
    for got, m in zip(y, x.float()):
        ref, _ = tokens.orthogonalize(m.double().numpy(), C32, 5, float(np.float32(EPS)))
        own += np.sum((got - ref) ** 2)
        plain += np.sum((in_fp32(m).double().numpy() - ref) ** 2)
        size += np.sum(ref ** 2)
    own, plain = np.sqrt(own / size), np.sqrt(plain / size)
    print("%d of %d x %d: %.2e, in FP32 %.2e" % (B, R, C, own, plain))
    assert own <= FACTOR * plain, (own, plain)
