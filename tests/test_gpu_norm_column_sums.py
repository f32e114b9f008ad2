"""Gradients of gamma and beta over many samples of one row: terms that fp32 would round the same way again and again."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# U: one fp32 operation.  A workgroup's sums are rounded once; at most 32 row lanes and teams are added in fp32 before that, and the sums of all
# workgroups in 64 bits.
U, K = 2.0 ** -23, 32


def test_rows_by_themselves():
    """Of 8 M x 256 a thread has a thousand rows."""
    n, c = 1 << 23, 256
    x = torch.empty(n, c, device=DEV).normal_()
    dy = torch.full((n, c), 1 + 0.99 * 2.0 ** -15, device=DEV)
    mean, rstd = torch.zeros(n, 1, device=DEV), torch.ones(n, 1, device=DEV)
    dgamma, dbeta = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, 1, n, True), device=DEV, dtype=torch.uint8)
    gnn.gnn_group_norm_bwd(x, None, None, mean, rstd, dy, None, dgamma, dbeta, 1, n_samples=n, workspace=ws)
    torch.cuda.synchronize()
    want = n * float(dy[0, 0])
    assert float((dbeta.double() - want).abs().max()) <= U * K * want
    terms = torch.zeros(c, device=DEV, dtype=torch.float64)
    size = torch.zeros_like(terms)
    for part in x.split(1 << 20):
        terms += part.double().sum(0) * float(dy[0, 0])
        size += part.double().abs().sum(0)
    assert bool(((dgamma.double() - terms).abs() <= U * K * size).all())


@pytest.mark.parametrize("hint", [0, 1])
@pytest.mark.parametrize("n,c,dtype", [(1 << 23, 4, torch.float32), (1 << 22, 8, torch.bfloat16), (1 << 20, 20, torch.float32)])
def test_samples_of_one_row(n, c, dtype, hint):
    """Adding 1 + 0.99 / 2^15 to sums from 512 on drops half a unit of their last place each time."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n + c)
    x = torch.empty(n, c, device=DEV).normal_(generator=gen).to(dtype)
    # (bf16 has no such number; 1 + 2^-7 loses as much from 2^17 on, and less before)
    dy = torch.full((n, c), 1 + 0.99 * 2.0 ** -15 if dtype == torch.float32 else 1 + 2.0 ** -7, device=DEV).to(dtype)
    ptr = torch.arange(n + 1, device=DEV, dtype=torch.int32)
    gamma, beta = torch.ones(c, device=DEV), torch.zeros(c, device=DEV)
    mean, rstd = torch.empty(n, 1, device=DEV), torch.empty(n, 1, device=DEV)
    dgamma, dbeta = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, 1, n, True), device=DEV, dtype=torch.uint8)
    more = dict(sample_ptr=ptr, workspace=ws, max_sample_rows=hint)
    gnn.gnn_group_norm_fwd(x, gamma, beta, torch.empty_like(x), mean, rstd, 1, **more)
    gnn.gnn_group_norm_bwd(x, gamma, beta, mean, rstd, dy, None, dgamma, dbeta, 1, **more)
    torch.cuda.synchronize()
    want = n * float(dy[0, 0])
    assert float((dbeta.double() - want).abs().max()) <= U * K * want
    xh = (x.double() - mean) * rstd.double()
    terms = xh * dy.double()
    # a term is off by its mean's and deviation's distances and two operations
    size = (terms.abs() + (mean.abs() * rstd).double() * dy.double()).sum(0)
    assert bool(((dgamma.double() - terms.sum(0)).abs() <= U * K * size).all())
