"""BF16 results of the orthogonalisation where a matrix has little in most directions: the last product's operands are large there (up to a^3 = 41 for the polynomial of three
steps), so that whatever they are rounded to counts that many times in the few directions that the matrix has.

How far a result may be off: test_gpu_ortho.py has what the iteration itself may be (`allowed`, of the result's norm).  The result is then rounded once.  How far a rounding takes a value
is its distance to the nearest of BF16's numbers, which changes by no more than the value does: the roundings' norm is that of the exact result's own roundings and `allowed` at most."""
import numpy as np
import pytest
import torch

from jzt_blocks import DEV, wide
from oracle import tokens
from test_gpu_ortho import C32, EPS, allowed, jz, run    # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def low_rank(R, C, rank, noise, B=2):
    g = np.random.default_rng([1, R, C, rank])
    x = g.standard_normal((B, R, rank)) @ g.standard_normal((B, rank, C)) + noise * g.standard_normal((B, R, C))
    return torch.from_numpy(x).float().to(DEV)


# the shorter side at most 128; beyond it, with steps in its space (elongated ones); with steps of X itself
@pytest.mark.parametrize("R,C", [(100, 140), (128, 512), (300, 70), (256, 2048), (1500, 150), (300, 310), (520, 500)])
@pytest.mark.parametrize("rank,noise", [(1, 0.0), (3, 0.0), (4, 1e-4)])
@pytest.mark.parametrize("steps", [1, 3, 5])
def test_matrices_of_low_rank(jz, R, C, rank, noise, steps):
    x = low_rank(R, C, rank, noise)
    y = run(jz, x, torch.bfloat16, steps)
    for got, m in zip(wide(y), wide(x)):
        ref, norms = tokens.orthogonalize(m, C32, steps, float(np.float32(EPS)))
        size = np.linalg.norm(ref)
        own = np.linalg.norm(torch.from_numpy(ref).to(torch.bfloat16).double().numpy() - ref) / size
        off = np.linalg.norm(got - ref) / size
        assert off <= own + 2 * allowed(norms), (off, own, allowed(norms))


@pytest.mark.parametrize("B,R,C,steps", [(1, 9, 1, 1), (3, 100, 140, 1), (2, 150, 260, 1), (1, 2100, 130, 1), (1, 600, 590, 1), (1, 600, 590, 5), (3, 300, 260, 4), (16, 900, 880, 5), (1, 2700, 2690, 2)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16])
def test_results_are_rounded_once(jz, B, R, C, steps, out):
    """Products and sums are the same whatever the result's type is, where the steps are those of X itself, and the factor behind them is a power of two: a 16-bit result is the FP32 one, rounded to nearest."""
    x = low_rank(R, C, 3, 0.3, B)
    assert torch.equal(run(jz, x, out, steps), run(jz, x, torch.float32, steps).to(out))
