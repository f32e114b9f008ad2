"""The gradient of a table on each of its ways: one launch, counted places, sorted ids in short and long runs, tables of the sort that are scanned."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = 2.0 ** -24


def gradient(ids, dy, v, dtype=F32, **kw):
    dt = torch.full((v, dy.shape[1]), float("nan"), device=DEV, dtype=dtype)
    ws = torch.full((gnn.gnn_lookup_workspace_bytes(v, len(ids), dy.shape[1]),), 255, device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids.to(DEV), dy.to(DEV), dt, workspace=ws, **kw)
    return dt.cpu().double()


def sums(ids, dy, v):
    there = (ids >= 0) & (ids < v)
    return [torch.zeros(v, dy.shape[1], dtype=torch.float64).index_add_(0, ids[there], x[there].double()) for x in (dy, dy.abs())]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("share", [0.05, 0.5, 0.98])
@pytest.mark.parametrize("n,v", [(1000, 300), (5000, 300), (5000, 40000), (50000, 700), (150000, 47), (150000, 60000)])
def test_rows_of_ids_that_name_none_do_not_matter(n, v, share, types):
    """Not finite, first and last among them, on every way."""
    gen = torch.Generator().manual_seed(n + v)
    ids, dy = torch.randint(0, v, (n,), generator=gen), torch.randn(n, 12, generator=gen).to(types[1])
    none = torch.rand(n, generator=gen) < share
    none[0] = none[n - 1] = True
    ids[none] = torch.where(torch.rand(n, generator=gen) < 0.5, -1, v)[none]
    dy[none] = torch.tensor([float("nan"), float("inf"), -float("inf")])[torch.randint(0, 3, (n,), generator=gen)][:, None].expand(n, 12)[none].to(types[1])
    got = gradient(ids, dy, v, types[0], scale=0.5)
    want, size = sums(ids, torch.where(none[:, None], 0.0, dy.float()), v)
    assert torch.isfinite(got).all()
    assert ((got - 0.5 * want).abs() <= 0.5 * (34 * HALF * size + (2.0 ** -8 if types[0] == BF16 else 0.0) * 1.01 * size)).all()
