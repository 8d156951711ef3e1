"""Kernels of the residual-block operators that a rule on sizes chooses, each at sizes that reach it, against the formulas in 64 bits with the checks and tolerances of
the other tests (test_gpu_ffn.py, test_gpu_norm_residual.py, imported from there)."""
import pytest
import torch

import test_gpu_ffn as ffn
import test_gpu_norm_residual as norm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jz():
    from paper_1807_11205_amd import api
    api.lib()
    assert torch.cuda.is_available()
    return api


# Few rows: eight wavefronts a workgroup up to 4096 columns of a product, four above; where rows are not on 16 bytes 16, 8 (from 4097 columns) and 4 (from 8193).
@pytest.mark.parametrize("M", [1, 16, 20, 40, 64])
@pytest.mark.parametrize("D, F, O", [(64, 4096, 64), (64, 4104, 64), (128, 5632, 72), (64, 8200, 64), (64, 12288, 64), (200, 64, 4104), (64, 72, 8200), (320, 4112, 5640)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_rows_of_many_columns(jz, M, D, F, O, dtype):
    c = ffn.Case(jz, M, D, F, O, dtype, "gelu_tanh")
    c.forward()
    c.check_forward()


@pytest.mark.parametrize("M", [1, 20, 40])
@pytest.mark.parametrize("D, F, O", [(63, 4096, 65), (65, 4101, 64), (64, 5637, 64), (130, 8193, 33), (61, 8197, 64), (64, 66, 4101), (99, 67, 8209), (33, 4111, 5633)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_rows_of_many_columns_at_any_alignment(jz, M, D, F, O, dtype):
    c = ffn.Case(jz, M, D, F, O, dtype, "silu")
    c.forward()
    c.check_forward()


# What a plan may be: 256 x 256 or 128 x 128 tiles, whole or with shared sums, for each product.  The smallest sizes found for each; test_launch_sizes.py says that they
# still reach it.  The epilogue of dh has every activation's own form, in each tile and behind shared sums.
LARGE_DH, LARGE_DH_SHARED, SMALL_DH_SHARED = (7536, 8, 1928, 648), (7048, 56, 2464, 2552), (136, 8, 8, 696)


@pytest.mark.parametrize("act", list(ffn.ACTS))
@pytest.mark.parametrize("size, dtype", [(LARGE_DH, "f16"), ((7535, 9, 1927, 650), "bf16"), (SMALL_DH_SHARED, "bf16"), (SMALL_DH_SHARED, "f16")])
def test_derivatives_of_every_activation(jz, act, size, dtype):
    ffn.Case(jz, *size, dtype, act).check()


@pytest.mark.parametrize("act, dtype", [("gelu", "f16"), ("gelu_tanh", "bf16"), ("relu", "f16"), ("silu", "bf16")])
def test_derivatives_behind_shared_sums_of_large_tiles(jz, act, dtype):
    ffn.Case(jz, *LARGE_DH_SHARED, dtype, act).check()


@pytest.mark.parametrize("size", [(2240, 2120, 3664, 16), (968, 120, 7032, 4192), (8136, 136, 5944, 152), (8272, 416, 3640, 40), (2239, 2119, 3663, 17), (8135, 135, 5943, 151)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_shared_sums_of_large_tiles(jz, size, dtype):
    ffn.Case(jz, *size, dtype, "silu").check()


@pytest.mark.parametrize("size", [(136, 672, 8, 8), (80, 8, 696, 8), (72, 728, 8, 488), (672, 8, 8, 8), (152, 8, 360, 8), (672, 9, 7, 11)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_shared_sums_of_small_tiles(jz, size, dtype):
    ffn.Case(jz, *size, dtype, "gelu").check()


# Gates that change inside a slab of rows, in workgroups of 128 to 1024 lanes: parameters in registers, in LDS, and read again for every row
@pytest.mark.parametrize("C", [513, 1001, 1024, 2048, 2049, 4096, 4097, 8192, 8200, 16383])
@pytest.mark.parametrize("per", [1, 3, 7])
@pytest.mark.parametrize("dtype, res", [("bf16", "f32"), ("f16", None)])
def test_gates_that_change_inside_a_slab(jz, C, per, dtype, res):
    c = norm.Case(jz, 42, C, dtype, res, per=per, seed=11)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()


@pytest.mark.parametrize("C", [1001, 4100, 9000])
@pytest.mark.parametrize("post, pre", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("per", [0, 5])
def test_parts_of_wide_rows(jz, C, post, pre, per):
    c = norm.Case(jz, 35, C, "f16", "f32", per=per, post=post, pre=pre, seed=12)
    c.forward()
    c.check_forward()
    c.backward()
    c.check_backward()
