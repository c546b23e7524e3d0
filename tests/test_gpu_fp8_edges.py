"""The 8-bit decoder operators on the GPU at the ends of their ranges: last tiles of one
row, sequences beyond their table, weights far below the largest, values that are no
numbers. Definitions in 64 bits and tolerances as in test_gpu_fp8.
"""
import math

import pytest
import torch

from .test_gpu_fp8 import (BF16, DEV, E4M3, E5M2, E8M0, F16, F32, filled_cache, near, normal, operands, product_terms,  # noqa: F401
                           value)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_1905_13298_amd import ops as o
    return o


# ---------------------------------------------------------------------------
# Product.

@pytest.mark.parametrize("m,n", [(65, 65), (1025, 2049), (2177, 2049), (3841, 3841)])
@pytest.mark.parametrize("k", [1, 16, 100, 128, 272])
def test_product_tiles_of_one_row(ops, m, n, k):
    """Last tiles of one row of x and of w (tiles of 64, of 128 in four and in two stages, of 256), with
    fewer steps than a tile sends for ahead: their buffers are a row, shorter than those steps' offsets."""
    x8, xs, w8, ws = operands(ops, m, n, k, E4M3, k)
    y = ops.linear_fp8(x8, xs, w8, ws).cpu()
    rows = torch.tensor([0, 1, m // 2, m - 2, m - 1])
    x, w = value(x8, xs)[rows], value(w8, ws, 128)
    near(y[rows], x @ w.T, product_terms(x, w, k, False))
