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
