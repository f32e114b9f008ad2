"""Group norm of matrices so large that a test looks at some of their rows, and at the sums of all on the device."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, K = 2.0 ** -23, 32  # one fp32 operation; how many of them a result has, as in test_gpu_norm.py
HALF_BF16 = 2.0 ** -8


@pytest.fixture(autouse=True)
def memory():
    """Large tensors go back to the device, which has no room for two tests' at once."""
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def need(nbytes):
    free = torch.cuda.mem_get_info()[0]
    if free < nbytes + (2 << 30):
        pytest.skip(f"{nbytes / 2 ** 30:.0f} GiB of device memory")


def chunks(n, c):
    step = max(1, (1 << 27) // c)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def forward(x, groups, samples, y, act=gnn.GNN_ACT_NONE, **kw):
    n, c = x.shape
    mean, rstd = (torch.empty(samples, groups, device=DEV) for _ in range(2))
    ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, groups, samples), device=DEV, dtype=torch.uint8)
    gnn.gnn_group_norm_fwd(x, None, None, y, mean, rstd, groups, n_samples=samples, act=act, workspace=ws, **kw)
    torch.cuda.synchronize()
    return mean, rstd


def test_more_samples_than_a_dimension_of_a_grid_has_threads_for():
    """300 M rows of three values, each normalised by itself: sixteen threads a sample at least."""
    n, c = 300_000_000, 3
    x = torch.empty(n, c, device=DEV).normal_()
    y = torch.full_like(x, float("nan"))
    mean, rstd = forward(x, 1, n, y)
    for a, b in chunks(n, c):
        v = x[a:b].double()
        m = v.mean(1, keepdim=True)
        d = v - m
        r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
        assert bool(((mean[a:b] - m).abs() <= U * K * v.abs().mean(1, keepdim=True)).all()), a
        assert bool(((rstd[a:b] - r).abs() <= U * K * r).all()), a
        assert bool(((y[a:b] - d * r).abs() <= U * K * (1 + (d * r).abs())).all()), a


def test_more_rows_by_themselves_than_a_dimension_of_a_grid_has_threads_for():
    """2^28 rows of 136 bf16 values, sixteen threads each; rows of zeros but for a few."""
    n, c = (1 << 28) + 5, 136
    need(2 * 2 * n * c + 24 * n)
    x, y = (torch.empty(n, c, device=DEV, dtype=torch.bfloat16) for _ in range(2))
    x.zero_()
    rows = torch.tensor(sorted({0, 1, 1000, (1 << 27) - 1, 1 << 27, (1 << 27) + 9, (1 << 28) - 17, (1 << 28) - 1, 1 << 28, n - 2, n - 1}), device=DEV)
    x[rows] = torch.randn(len(rows), c, device=DEV).bfloat16()
    y.fill_(float("nan"))
    mean, rstd = forward(x, 1, n, y)
    v = x[rows].double()
    d = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + 1e-5)
    assert bool(((rstd[rows] - r).abs() <= U * K * r).all())
    assert bool(((y[rows].double() - d * r).abs() <= U * K * (1 + (d * r).abs()) + HALF_BF16 * (d * r).abs()).all())
    y[rows] = 0
    assert not any(bool(y[a:b].any()) for a, b in chunks(n, c))  # (NaN is true)


def test_more_vectors_than_a_dimension_of_a_grid_has_threads_for():
    """Four samples of 2^23 rows of 1,024 values: results are written by threads of two vectors."""
    rows, c, groups = (1 << 23) + 16, 1024, 8
    n = 4 * rows
    need(2 * 4 * n * c + (1 << 30))
    x, y = (torch.empty(n, c, device=DEV) for _ in range(2))
    for i, (a, b) in enumerate(chunks(n, c)):
        x[a:b].normal_()
    mean, rstd = forward(x, groups, 4, y)
    for s in range(4):
        total, squares = torch.zeros(groups, device=DEV, dtype=torch.float64), torch.zeros(groups, device=DEV, dtype=torch.float64)
        for a, b in chunks(rows, c):
            v = x[s * rows + a:s * rows + b].view(b - a, groups, -1).double()
            total += v.sum((0, 2))
            squares += (v * v).sum((0, 2))
        count = rows * (c // groups)
        m = total / count
        r = 1 / torch.sqrt(squares / count - m * m + 1e-5)
        assert bool(((mean[s] - m).abs() <= U * K).all()) and bool(((rstd[s] - r).abs() <= U * K * r).all()), s
        at = torch.tensor([s * rows, s * rows + rows // 2 + 3, (s + 1) * rows - 1], device=DEV)
        want = ((x[at].view(3, groups, -1).double() - m[:, None]) * r[:, None]).view(3, c)
        assert bool(((y[at] - want).abs() <= U * K * (1 + want.abs())).all()), s
