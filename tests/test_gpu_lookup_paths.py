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


# Roundings of a sum in fp32 on its way: in one launch that of the sum, which is made in 64 bits; else those of a run's additions (7 of 8 positions, 31 of 32), of the
# two parts that workgroups hand on, and of the sum.  Then the product with the scale.
@pytest.mark.parametrize("kind", ["uniform", "hubs", "one", "stretches"])
@pytest.mark.parametrize("n,v,roundings", [(2048, 256, 2), (2048, 255, 11), (2049, 5000, 11), (6143, 5000, 11), (6144, 5000, 11), (6145, 5000, 11), (6145, 300000, 11),
                                           (65536, 3000, 11), (65537, 3000, 11), (131071, 3000, 11), (131072, 3000, 35), (262144, 3000, 35), (262145, 70000, 35)])
def test_sums_are_as_close_as_their_way_allows(n, v, roundings, kind):
    gen = torch.Generator().manual_seed(n)
    if kind == "uniform":
        ids = torch.randint(-1, v, (n,), generator=gen)
    elif kind == "hubs":
        ids = (torch.rand(n, generator=gen, dtype=torch.float64) ** 4 * v).long()
    elif kind == "one":
        ids = torch.full((n,), v - 1)
    else:  # of 1 to 300 positions, in any order
        ids = torch.repeat_interleave(torch.arange(n), torch.randint(1, 300, (n,), generator=gen))[:n].clamp(max=v)[torch.randperm(n, generator=gen)]
    dy = torch.randn(n, 20, generator=gen)
    scale = float(torch.tensor(0.3))
    want, size = sums(ids, dy, v)
    got = gradient(ids, dy, v, scale=scale)
    assert ((got - scale * want).abs() <= scale * HALF * 1.01 * ((roundings - 2) * size + 2 * want.abs() + 2.0 ** -20 * size)).all()


def test_positions_whose_digits_are_scanned_and_gradients_beyond_32_bits_of_offsets():
    """More than 4,096 tiles of the sort in all of its passes, and more than 2^32 values; whole numbers, so that every sum is exact."""
    n, v, f = 16900000, 2000003, 256
    assert n > 4096 * 4096 and n * f > 1 << 32
    gen = torch.Generator(device=DEV).manual_seed(8)
    ids = torch.randint(-1, v + 1, (n,), device=DEV, generator=gen, dtype=torch.int32)
    ids[-1], ids[0] = v - 1, 0
    dy = torch.empty(n, f, device=DEV, dtype=BF16)
    want = torch.zeros(v + 2, f, device=DEV)
    for part in range(0, n, 1 << 19):
        x = torch.randint(-8, 9, (min(n, part + (1 << 19)) - part, f), device=DEV, generator=gen, dtype=torch.int8)
        dy[part:part + len(x)] = x.to(BF16)
        want.index_add_(0, ids[part:part + len(x)].long() + 1, x.float())
    dt = torch.full((v, f), float("nan"), device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, dy, dt, workspace=ws)
    assert torch.equal(dt, want[1:v + 1])
