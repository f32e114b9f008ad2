"""Group norm of many samples of more columns than a workgroup has at once: slices of whole groups, groups in pieces, narrow last slices."""
import numpy as np
import pytest
import torch

from test_gpu_norm import check
from test_gpu_norm_statistics import KINDS, check as check_statistics, unlike

pytestmark = pytest.mark.gpu
# columns and groups: slices of four groups and one more; of 1,024 and 1; of 512 groups of two and one more; a group in two pieces, in three; many of 1,025
SHAPES = [(1030, 5), (1025, 1025), (1026, 513), (1025, 1), (3001, 1), (4100, 4), (2050, 2)]


@pytest.mark.parametrize("c,groups", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ragged_samples(c, groups, dtype):
    # a tile has 16,384 values: 5 to 16 rows
    sizes = [16, 1, 15, 17, 16, 0, 3, 0, 13, 40, 8, 0, 0, 2, 1, 1, 33, 16, 100, 5, 0]
    ptr = [0] + [int(v) for v in np.cumsum(sizes)]
    for act, ptr_dtype in (("silu", torch.int64), ("relu", torch.int32)):
        print("wide", c, groups, dtype, act, flush=True)
        check(ptr[-1], c, groups, ptr, act, dtype, ptr_dtype=ptr_dtype)
    # more samples than tiles
    ptr = [0] + [int(v) for v in np.cumsum(np.random.default_rng(5).integers(0, 4, 400))]
    check(ptr[-1], c, groups, ptr, "silu", dtype)


@pytest.mark.parametrize("c,groups", SHAPES)
def test_strides_and_equal_samples(c, groups):
    check(330, c, groups, list(range(0, 331, 110)), "silu", uniform=1, lds=(c + 3, c + 1, c + 5), front=3)
    check(330, c, groups, list(range(0, 331, 110)), "none", torch.bfloat16, uniform=1, affine=False)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("c,groups", [(1025, 1), (3001, 1), (1026, 513)])
def test_a_row_unlike_the_rest(kind, c, groups):
    ptr = [0, 1, 61, 64, 64, 130, 200]
    x = torch.cat([unlike(kind, b - a, c, a + c) for a, b in zip(ptr, ptr[1:])])
    x[61:64, :7] += 500  # columns unlike the rest of their group
    check_statistics(x, groups, kind, ptr, rounded=False)


@pytest.mark.parametrize("c,groups,dtype", [(8004, 4, torch.bfloat16), (8190, 9, torch.bfloat16), (4086, 9, torch.float32)])
def test_few_rows_in_many_samples(c, groups, dtype):
    """A workgroup's sums and parameters are more than 64 KB there."""
    for rows in (1, 3, 9):
        print("few rows", rows, c, groups, dtype, flush=True)
        check(260 * rows, c, groups, list(range(0, 260 * rows + 1, rows)), "silu", dtype, uniform=1)
