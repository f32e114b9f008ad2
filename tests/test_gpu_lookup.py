"""Rows of a table by id, and the gradient of the table, against the formulas in 64 bits."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # half a step, relative
# A sum: at most 64 terms one after the other in fp32 (63 roundings of sums that |x| bounds), the parts that are joined in fp64 rounded to fp32 on their way
# through LDS, workgroups and the result (3), and the product with the scale (1).
SUM = 70 * 2.0 ** -24


def make_ids(n, v, kind, gen, dtype):
    if kind == "uniform":
        ids = torch.randint(0, max(v, 1), (n,), generator=gen)
    elif kind == "hubs":
        ids = (torch.rand(n, generator=gen, dtype=torch.float64) ** 4 * v).long().clamp(max=v - 1)
    elif kind == "one":
        ids = torch.full((n,), v // 2)
    elif kind == "two":  # the first and the last row
        ids = torch.where(torch.rand(n, generator=gen) < 0.5, 0, v - 1)
    elif kind == "sorted":
        ids = torch.arange(n) * max(v, 1) // max(n, 1)
    elif kind == "none":
        ids = torch.full((n,), -1)
    else:  # some that name no row, on either side and beyond 32 bits
        ids = torch.randint(-v, 2 * v, (n,), generator=gen)
        if dtype == torch.int64:
            ids[::7] += 1 << 32
    return ids.to(dtype)


def rows_of(gen, n, f, dtype, stride):
    return torch.randn(n, stride, generator=gen).to(dtype).to(DEV)[:, :f]


SHAPES = [  # v, n, f, ids
    (1, 1, 1, "uniform"), (1, 300, 3, "uniform"), (5, 1, 4, "uniform"), (47, 1000, 7, "odd"), (300, 31, 8, "uniform"), (300, 33, 12, "sorted"),
    (4096, 1021, 64, "uniform"), (4096, 257, 100, "hubs"), (257, 5000, 100, "hubs"), (2, 3000, 257, "two"), (1000, 2000, 602, "odd"), (7, 9000, 20, "one"),
    (512, 512, 33, "none"), (100000, 3, 5, "uniform"), (33, 4000, 1030, "hubs")]


@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_by_id(shape, types):
    v, n, f, kind = shape
    gen = torch.Generator().manual_seed(v + n + f)
    ids = make_ids(n, v, kind, gen, torch.int64 if f % 2 else torch.int32)
    table = rows_of(gen, v, f, types[0], f + (f % 3))
    y = torch.full((n, f + 5), float("nan"), device=DEV, dtype=types[1])
    scale = 0.3
    gnn.gnn_lookup_fwd(table, ids.to(DEV), y[:, :f], scale=scale)
    at = ids.long()
    there = (at >= 0) & (at < v)
    want = table.cpu().double()[at.clamp(0, v - 1)] * float(torch.tensor(scale)) * there[:, None]
    got = y.cpu().double()
    # the product is rounded to fp32, then to Y's type
    assert ((got[:, :f] - want).abs() <= (2.0 ** -24 + HALF[types[1]]) * 1.01 * want.abs()).all()
    assert torch.isnan(got[:, f:]).all()  # columns behind the row are left
    assert not got[:, :f][~there].any()


def reference(ids, dy, v, scale):
    at = ids.long()
    there = (at >= 0) & (at < v)
    x = dy.cpu().double()[there]
    zero = torch.zeros(v, dy.shape[1], dtype=torch.float64)
    s = float(torch.tensor(scale))
    return zero.index_add(0, at[there], x) * s, zero.index_add(0, at[there], x.abs()) * abs(s)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient_of_the_table(shape, types, accumulate):
    v, n, f, kind = shape
    gen = torch.Generator().manual_seed(v + n + f)
    ids = make_ids(n, v, kind, gen, torch.int64 if f % 2 else torch.int32)
    dy = rows_of(gen, n, f, types[1], f + (f % 3))
    start = torch.randn(v, f, generator=gen).to(types[0]).to(DEV)
    dt = torch.full((v, f + 5), float("nan"), device=DEV, dtype=types[0])
    if accumulate:
        dt[:, :f] = start
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids.to(DEV), dy, dt[:, :f], scale=-0.7, accumulate=accumulate, workspace=ws)
    want, size = reference(ids, dy, v, -0.7)
    if accumulate:
        want = want + start.cpu().double()
    got = dt.cpu().double()
    # with accumulate the sum is rounded to fp32 before it is to the table's type
    bound = SUM * size + (HALF[types[0]] + (2.0 ** -24 if accumulate else 0)) * 1.01 * want.abs()
    assert ((got[:, :f] - want).abs() <= bound + SUM * HALF[types[0]] * size).all()
    assert torch.isnan(got[:, f:]).all()
    untouched = size.sum(1) == 0
    if accumulate:
        assert torch.equal(dt[:, :f].cpu()[untouched], start.cpu()[untouched])
    else:
        assert not got[:, :f][untouched].any()
    again = dt.clone()
    if accumulate:
        again[:, :f] = start
    gnn.gnn_lookup_bwd(ids.to(DEV), dy, again[:, :f], scale=-0.7, accumulate=accumulate, workspace=ws)
    assert torch.equal(again[:, :f], dt[:, :f])  # reproducible to the bit


@pytest.mark.parametrize("n", [31, 32, 33, 63, 64, 65, 255, 256, 257, 511, 512, 513, 4095, 4096, 4097, 8193, 70000])
@pytest.mark.parametrize("f", [64, 256])
def test_sums_that_end_where_runs_and_workgroups_end(n, f):
    """Ids in long stretches whose ends lie at and beside the ends of runs of 32 positions and of workgroups' positions."""
    gen = torch.Generator().manual_seed(n)
    cuts = sorted({c for c in (1, 31, 32, 33, 64, 127, 128, 129, 256, 384, 512, 1024, 2049, 4096, 8192, 40000) if c < n})
    ids = torch.zeros(n, dtype=torch.int64)
    for c in cuts:
        ids[c:] += 1
    dy = torch.randn(n, f, generator=gen).to(DEV)
    v = len(cuts) + 1
    order = torch.randperm(n, generator=gen)
    for perm in (torch.arange(n), order):
        dt = torch.empty(v, f, device=DEV)
        ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)
        gnn.gnn_lookup_bwd(ids[perm].to(DEV), dy, dt, workspace=ws)
        want, size = reference(ids[perm], dy, v, 1.0)
        assert ((dt.cpu().double() - want).abs() <= SUM * size + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("n,f", [(131072, 16), (150001, 100), (200003, 3), (131073, 260)])
def test_long_and_short_sums_of_many_positions(n, f, types, accumulate):
    """Sums of one to some thousand rows side by side, whose positions in the sorted list begin and end at and beside whole runs of 32."""
    gen = torch.Generator().manual_seed(n)
    lengths = torch.tensor([0, 0, 1, 1, 1, 2, 3, 31, 32, 33, 61, 62, 63, 64, 65, 95, 96, 97, 255, 256, 257, 1000, 5000])
    rows = lengths[torch.randint(0, len(lengths), (n,), generator=gen)]
    rows = rows[:int((rows.cumsum(0) < n - 40).sum())]
    v = max(len(rows) + 300, n // 20)
    ids = torch.repeat_interleave(torch.arange(len(rows)), rows)
    ids = torch.cat([ids, torch.full((20,), -1), torch.full((n - 20 - len(ids),), v - 1)])
    ids = ids[torch.randperm(n, generator=gen)]
    dy = torch.randn(n, f, generator=gen).to(types[1]).to(DEV)
    dt = torch.full((v, f), 3.0, device=DEV, dtype=types[0])
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)
    for _ in range(2):
        dt.fill_(3.0)
        ws.fill_(255)
        gnn.gnn_lookup_bwd(ids.to(DEV), dy, dt, scale=0.5, accumulate=accumulate, workspace=ws)
        want, size = reference(ids, dy, v, 0.5)
        want = want + 3.0 if accumulate else want
        bound = SUM * size + (HALF[types[0]] + (2.0 ** -24 if accumulate else 0)) * 1.01 * want.abs() + SUM * HALF[types[0]] * size
        assert ((dt.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("n,v", [(131072, 4096), (131072, 5000000), (200000, 200000)])
def test_tables_of_other_sizes_than_the_ids(n, v):
    gen = torch.Generator().manual_seed(n + v)
    for kind in ("uniform", "hubs", "one", "none"):
        ids = make_ids(n, v, kind, gen, torch.int32)
        dy = torch.randn(n, 8, generator=gen).to(DEV)
        dt = torch.full((v, 8), float("nan"), device=DEV)
        ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, 8), device=DEV, dtype=torch.uint8)
        gnn.gnn_lookup_bwd(ids.to(DEV), dy, dt, scale=float("inf") if kind == "none" else 1.0, workspace=ws)
        want, size = reference(ids, dy, v, 1.0)
        assert ((dt.cpu().double() - want).abs() <= SUM * size + 2.0 ** -24 * want.abs()).all(), kind


def test_what_names_no_row_is_not_read():
    """NaN and infinities in rows whose id names none, and in rows of the table that no id names."""
    ids = torch.tensor([0, -1, 2, 5, 2], dtype=torch.int32, device=DEV)
    dy = torch.ones(5, 8, device=DEV)
    dy[1], dy[3] = float("nan"), float("inf")
    dt = torch.empty(4, 8, device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(4, 5, 8), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, dy, dt, workspace=ws)
    assert dt[:, 0].tolist() == [1.0, 0.0, 2.0, 0.0]
    table = torch.ones(4, 8, device=DEV)
    table[1] = float("nan")
    y = torch.empty(5, 8, device=DEV)
    gnn.gnn_lookup_fwd(table, ids, y, scale=2.0)
    assert y[:, 0].tolist() == [2.0, 0.0, 2.0, 0.0, 2.0]
    # accumulate does not touch a row that no id names, NaN or not
    dt = torch.full((4, 8), float("nan"), device=DEV)
    dt[0] = dt[2] = 1.0
    gnn.gnn_lookup_bwd(ids, dy, dt, accumulate=True, workspace=ws)
    assert dt[0, 0] == 2.0 and dt[2, 7] == 3.0 and torch.isnan(dt[1]).all() and torch.isnan(dt[3]).all()


def test_empty_calls():
    table, none = torch.ones(4, 8, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    gnn.gnn_lookup_fwd(table, none, torch.empty(0, 8, device=DEV))
    dt = torch.ones(300, 8, device=DEV)
    gnn.gnn_lookup_bwd(none, torch.empty(0, 8, device=DEV), dt, accumulate=True)
    assert (dt == 1).all()
    gnn.gnn_lookup_bwd(none, torch.empty(0, 8, device=DEV), dt)
    assert (dt == 0).all()
    y = torch.ones(3, 8, device=DEV)
    gnn.gnn_lookup_fwd(torch.empty(0, 8, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV), y)
    assert (y == 0).all()


def test_gradient_against_differences():
    """The gradient is that of sum dY Y: a step of one entry of the table changes it by the step times the gradient."""
    gen = torch.Generator().manual_seed(5)
    ids = torch.randint(0, 9, (40,), generator=gen).to(DEV)
    table, dy = torch.randn(9, 6, generator=gen).to(DEV), torch.randn(40, 6, generator=gen).to(DEV)
    dt = torch.empty(9, 6, device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(9, 40, 6), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, dy, dt, scale=0.5, workspace=ws)

    def value(t):
        y = torch.empty(40, 6, device=DEV)
        gnn.gnn_lookup_fwd(t, ids, y, scale=0.5)
        return float((y.double() * dy.double()).sum())
    for r, c in ((0, 0), (3, 5), (8, 2)):
        up, down = table.clone(), table.clone()
        up[r, c] += 1.0
        down[r, c] -= 1.0
        # linear: but for the rounding of 2 x 40 products of numbers below 8
        assert abs((value(up) - value(down)) / 2 - float(dt[r, c])) <= 80 * 8 * 8 * 2.0 ** -24


def test_other_streams_and_replays():
    gen = torch.Generator().manual_seed(3)
    v, n, f = 700, 5000, 100
    ids = make_ids(n, v, "hubs", gen, torch.int32).to(DEV)
    table, dy = torch.randn(v, f, generator=gen).to(DEV), torch.randn(n, f, generator=gen).to(DEV)
    y, dt = torch.empty(n, f, device=DEV), torch.empty(v, f, device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)

    def both(stream=None):
        gnn.gnn_lookup_fwd(table, ids, y, scale=0.5, stream=stream)
        gnn.gnn_lookup_bwd(ids, dy, dt, scale=0.5, workspace=ws, stream=stream)
    both()
    torch.cuda.synchronize()
    want = y.clone(), dt.clone()
    side = torch.cuda.Stream()
    y.fill_(float("nan")), dt.fill_(float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(dt, want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):  # with other ids in each replay
        ids.copy_(make_ids(n, v, "hubs" if k < 2 else "odd", gen, torch.int32))
        y.fill_(float("nan")), dt.fill_(float("nan")), ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone(), dt.clone()
        both()
        torch.cuda.synchronize()
        assert torch.equal(y, got[0]) and torch.equal(dt, got[1])


def test_a_table_beyond_32_bits_of_offsets():
    v, f = (1 << 32) // 512 + 1000, 512  # 4.3e9 elements of bf16
    table = torch.zeros(v, f, device=DEV, dtype=BF16)
    ids = torch.tensor([0, v - 1, v // 2, v - 1000], device=DEV)
    table[ids] = torch.arange(1, 5, device=DEV, dtype=BF16)[:, None]
    y = torch.empty(4, f, device=DEV)
    gnn.gnn_lookup_fwd(table, ids, y)
    assert torch.equal(y, torch.arange(1, 5, device=DEV)[:, None].expand(4, f).float())
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, 4, f), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, y, table, scale=2.0, workspace=ws)
    assert torch.equal(table[ids], 2 * y.to(BF16))
    assert float(table[1:v // 2].float().abs().amax()) == 0.0 and float(table[v // 2 + 1:v - 1000].float().abs().amax()) == 0.0


def test_the_widest_rows():
    f = 1 << 24
    gen = torch.Generator(device=DEV).manual_seed(17)
    ids = torch.tensor([2, -1, 0, 2, 2], device=DEV, dtype=torch.int32)
    dy = torch.randn(5, f, device=DEV, generator=gen)
    dt = torch.full((3, f), float("nan"), device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(3, 5, f), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, dy, dt, workspace=ws)
    assert torch.equal(dt[0], dy[2]) and not dt[1].any()
    want = dy[0].double() + dy[3].double() + dy[4].double()
    # two additions, each off by half a step of a sum that is at most the sum of the magnitudes
    assert ((dt[2].double() - want).abs() <= 2.02 * 2.0 ** -24 * (dy[0].abs() + dy[3].abs() + dy[4].abs())).all()
    y = torch.empty(5, f, device=DEV)
    gnn.gnn_lookup_fwd(dt, ids, y)
    assert torch.equal(y[0], dt[2]) and not y[1].any() and torch.equal(y[2], dt[0])


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("f", [1, 4, 33, 100, 260, 602])
@pytest.mark.parametrize("n,repeats", [(15, 1), (16, 16), (17, 17), (64, 31), (500, 32), (500, 33), (2047, 700), (2048, 2048), (2049, 2049)])
def test_sums_of_few_positions(n, repeats, f, types, accumulate):
    """One id `repeats` times among others, at random places."""
    gen = torch.Generator().manual_seed(n + f)
    v = max(600, n)
    ids = torch.randperm(v, generator=gen)[:n]
    ids[torch.randperm(n, generator=gen)[:repeats]] = 5
    ids[n // 3] = v + 1
    dy = rows_of(gen, n, f, types[1], f + 3)
    dtable = torch.randn(v, f + 1, generator=gen).to(types[0]).to(DEV)
    start = dtable.cpu().double()
    ws = torch.full((gnn.gnn_lookup_workspace_bytes(v, n, f),), 255, device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids.to(DEV), dy, dtable[:, :f], scale=0.5, accumulate=accumulate, workspace=ws)
    got = dtable.cpu().double()
    assert torch.equal(got[:, f], start[:, f])
    keep = ids < v
    want, size = torch.zeros(v, f, dtype=torch.float64), torch.zeros(v, f, dtype=torch.float64)
    d = dy.cpu().double()
    want.index_add_(0, ids[keep], 0.5 * d[keep])
    size.index_add_(0, ids[keep], 0.5 * d[keep].abs())
    if accumulate:
        want, size = want + start[:, :f], size + start[:, :f].abs()
    # SUM, a rounding of the sum with what was there, and that to the table's type
    assert ((got[:, :f] - want).abs() <= (SUM + 2.0 ** -24) * size + HALF[types[0]] * want.abs() * 1.01).all()
    if not accumulate:
        unnamed = torch.ones(v, dtype=torch.bool)
        unnamed[ids[keep]] = False
        assert (got[unnamed][:, :f] == 0).all()


@pytest.mark.parametrize("v", [262144, 262145, 1000003])
def test_few_positions_of_large_tables(v):
    gen = torch.Generator().manual_seed(v)
    ids = torch.randint(0, v, (100,), generator=gen)
    ids[:3] = torch.tensor([0, v - 1, v - 2])
    dy = torch.randn(100, 6, generator=gen).to(DEV)
    dtable = torch.full((v, 6), float("nan"), device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, 100, 6), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids.to(DEV), dy, dtable, scale=1.0, workspace=ws)
    want = torch.zeros(v, 6, dtype=torch.float64).index_add_(0, ids, dy.cpu().double())
    size = torch.zeros(v, 6, dtype=torch.float64).index_add_(0, ids, dy.cpu().double().abs())
    assert ((dtable.cpu().double() - want).abs() <= SUM * size).all()
    assert int((dtable != 0).any(1).sum()) == len(set(ids.tolist()))


@pytest.mark.parametrize("n,v,dtype", [(530000, 1000, F32), (1050001, 47, BF16), (1050000, 2000000, BF16)])
def test_whole_lines_beyond_the_caches(n, v, dtype):
    f = 128
    gen = torch.Generator(device=DEV).manual_seed(n)
    ids = torch.randint(-1, v, (n,), device=DEV, generator=gen)
    dy = torch.randn(n, f, device=DEV, generator=gen).to(dtype)
    assert n * f * dy.element_size() > 256 << 20
    dtable = torch.full((v, f), float("nan"), device=DEV)
    ws = torch.empty(gnn.gnn_lookup_workspace_bytes(v, n, f), device=DEV, dtype=torch.uint8)
    gnn.gnn_lookup_bwd(ids, dy, dtable, scale=1.0, workspace=ws)
    at = torch.where(ids < 0, v, ids)
    want, size = (torch.zeros(v + 1, f, device=DEV, dtype=torch.float64) for _ in range(2))
    for part in torch.arange(n, device=DEV).split(200000):
        want.index_add_(0, at[part], dy[part].double())
        size.index_add_(0, at[part], dy[part].double().abs())
    assert ((dtable.double() - want[:v]).abs() <= SUM * size[:v]).all()
