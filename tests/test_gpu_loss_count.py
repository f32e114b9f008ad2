"""The mean's divisor: counted in every workgroup or by a launch of its own, the same results and no long count beside short rows."""
import pytest
import torch

import paper_2104_06700_amd as gnn
from test_gpu_loss import check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n", [2047, 2048, 2049, 4095, 4096, 4097, 16384, 16385])
@pytest.mark.parametrize("c", [5, 47, 520])
def test_around_the_numbers_of_rows_that_are_counted_in_different_ways(n, c):
    check(n, c, labelled=0.3)
    check(n, c, torch.bfloat16, labelled=0.9, label_dtype=torch.int64)
    check(n, c if c < 500 else 1030, torch.bfloat16, labelled=0.002)


def time_of(call):
    for _ in range(5):
        call()
    times = []
    for _ in range(5):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(20):
            call()
        end.record()
        torch.cuda.synchronize()
        times.append(begin.elapsed_time(end) / 20 * 1e3)
    return min(times)


@pytest.mark.parametrize("n,c,dtype,label_dtype", [(16384, 520, torch.float32, torch.int32), (16384, 1030, torch.bfloat16, torch.int64), (8192, 520, torch.float32, torch.int64)])
def test_the_mean_takes_little_longer_than_the_sum(n, c, dtype, label_dtype):
    """Each of n workgroups that counts n labels reads many times what the rows have: 148 us instead of 31 for the first."""
    x = torch.randn(n, c, device=DEV).to(dtype)
    labels = torch.randint(0, c, (n,), device=DEV).to(label_dtype)
    loss, dx = torch.empty(1, device=DEV), torch.empty_like(x)
    ws = torch.empty(gnn.gnn_softmax_xent_workspace_bytes(n, c), device=DEV, dtype=torch.uint8)
    mean, total = (time_of(lambda: gnn.gnn_softmax_xent(x, labels, loss, dx, reduction=r, workspace=ws)) for r in (gnn.GNN_LOSS_MEAN, gnn.GNN_LOSS_SUM))
    assert mean <= 1.5 * total + 10, (mean, total)
