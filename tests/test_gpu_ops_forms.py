"""Forms of the calls of include/spec_ops.h that the size lists of test_gpu_ops.py do not come to."""
import numpy as np
import pytest
import torch

import ops_reference as ref
import paper_2504_00030_amd as pk
import test_gpu_ops as ops

pytestmark = pytest.mark.gpu

F8, F32, BF16 = ops.F8, ops.F32, ops.BF16


@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("K", [384, 400, 512, 656, 1040])
def test_product_in_tiles_of_128_by_128(K, y_dtype):
    """512 tiles, which fp32 results take in two stages and bf16 results in three, over three to nine blocks of k: rounds of the
    loop over the stages, and every number of steps that can be left behind it."""
    ops.test_product_launch_shapes(900, 8100, K, y_dtype)


@pytest.mark.parametrize("y_dtype", [F32, BF16])
@pytest.mark.parametrize("x_kind", [F32, BF16])
@pytest.mark.parametrize("R,N,K", [(8, 2048, 2048), (8, 5000, 2000), (24, 5000, 2000), (40, 5000, 1024), (113, 3100, 672)])
def test_product_of_wide_rows_in_both_result_types(R, N, K, x_kind, y_dtype):
    """One and two groups of columns by one to four tiles of rows that the product quantises itself."""
    ops._gemm_case(np.random.default_rng(R + N), R, N, K, x_kind, y_dtype, ldy_extra=4)
