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
    if free < nbytes + (4 << 30):
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


def sample_sums(per_row, ptr, a, b):
    """Sums over the rows a .. b-1 of each sample: differences of running sums, in 64 bits."""
    if len(ptr) == 2:
        return per_row.sum(0, keepdim=True)
    running = torch.cat([torch.zeros(per_row.shape[1], 1, device=DEV, dtype=torch.float64), per_row.t().contiguous().cumsum(1)], 1)
    at = ptr.long().clamp(a, b) - a
    return (running[:, at[1:]] - running[:, at[:-1]]).t()


def check(n, c, groups, dtype, act, samples=1, ptr=None, hint=0):
    """All statistics and sums over vertices, and the results of some rows, against the definition in 64 bits, part by part."""
    print("large", n, c, groups, dtype, act, samples, hint, flush=True)
    bf16 = dtype == torch.bfloat16
    acts = {"none": gnn.GNN_ACT_NONE, "silu": gnn.GNN_ACT_SILU}
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n + c)
    x, y, dy = (torch.empty(n, c, device=DEV, dtype=dtype) for _ in range(3))
    for a, b in chunks(n, c):
        x[a:b].normal_(generator=gen).mul_(1.5).add_(0.5)
        dy[a:b].normal_(generator=gen)
    y.fill_(float("nan"))
    gamma, beta = (1 + 0.2 * torch.randn(c, device=DEV, generator=gen), 0.3 * torch.randn(c, device=DEV, generator=gen))
    kw = dict(n_samples=samples, act=acts[act], max_sample_rows=hint)
    if ptr is not None:
        kw["sample_ptr"] = ptr
    else:
        ptr = torch.arange(samples + 1, device=DEV) * (n // samples)
    rows = (ptr[1:] - ptr[:-1]).long()
    member = torch.repeat_interleave(torch.arange(samples, device=DEV), rows, output_size=n)
    count = (rows * (c // groups)).clamp(min=1).double()[:, None]
    mean, rstd = (torch.full((samples, groups), float("nan"), device=DEV) for _ in range(2))
    ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, groups, samples, True), device=DEV, dtype=torch.uint8)
    gnn.gnn_group_norm_fwd(x, gamma, beta, y, mean, rstd, groups, workspace=ws, **kw)
    torch.cuda.synchronize()

    def part(a, b):
        return x[a:b].double().view(b - a, groups, -1)
    spans = chunks(n, c)
    m = sum(sample_sums(part(a, b).sum(2), ptr, a, b) for a, b in spans) / count
    spread = squares = 0
    for a, b in spans:
        d = part(a, b) - m[member[a:b]][:, :, None]
        squares = squares + sample_sums((d * d).sum(2), ptr, a, b)
        spread = spread + sample_sums(d.abs().sum(2), ptr, a, b)
    r = 1 / torch.sqrt(squares / count + 1e-5)
    assert bool(((mean - m).abs() <= U * m.abs() + U * K * spread / count + 1e-30).all()), "mean"
    assert bool(((rstd - r).abs() <= U * K * r).all()), "rstd"
    # some rows: the ends, and around powers of two and 2^31 values
    at = [0, 1, n // 3, n // 2, n - 2, n - 1] + [k + o for k in ((1 << 31) // c, (1 << 32) // c) if k + 1 < n for o in (-1, 0, 1)]
    at = torch.tensor(sorted(set(at)), device=DEV)
    g64, b64 = gamma.double(), beta.double()

    def normalised(xs, who, mean, rstd):
        xh = ((xs - mean[who][:, :, None]) * rstd[who][:, :, None]).view(-1, c)
        z = xh * g64 + b64
        return xh, z, torch.sigmoid(z)
    xh, z, sig = normalised(x[at].double().view(len(at), groups, -1), member[at], m, r)
    want, rough = (z * sig, 1.0) if act == "silu" else (z, 0.0)
    size = 1.1 * ((xh.abs() + 1) * g64.abs() + b64.abs()) + rough * want.abs() * z.abs()
    assert bool(((y[at].double() - want).abs() <= U * K * size + (HALF_BF16 * want.abs() if bf16 else 0)).all()), "y"
    assert not any(bool(torch.isnan(y[a:b]).any()) for a, b in spans)
    # backward, from the statistics as they are stored
    dx, dgamma, dbeta = y.fill_(float("nan")), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    gnn.gnn_group_norm_bwd(x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, groups, workspace=ws, **kw)
    torch.cuda.synchronize()
    m, r = mean.double(), rstd.double()

    def slopes(a, b):
        xh, z, sig = normalised(part(a, b), member[a:b], m, r)
        d = dy[a:b].double()
        dz = d * sig * (1 + z * (1 - sig)) if act == "silu" else d
        sxh = xh.abs() + (m * r).abs()[member[a:b]].repeat_interleave(c // groups, 1) + 1
        return xh, dz, sxh, dz.abs() + rough * d.abs() * (sxh * g64.abs() + b64.abs() + z.abs())
    want = [0, 0, 0, 0]
    s1 = s2 = a1 = a2 = 0
    for a, b in spans:
        xh, dz, sxh, sdz = slopes(a, b)
        want = [w + v for w, v in zip(want, (dz.sum(0), sdz.sum(0), (dz * xh).sum(0), (sdz * sxh).sum(0)))]
        s1, s2, a1, a2 = (s + sample_sums(v.view(b - a, groups, -1).sum(2), ptr, a, b) for s, v in
                          ((s1, dz * g64), (s2, dz * g64 * xh), (a1, sdz * g64.abs()), (a2, sdz * g64.abs() * sxh)))
    assert bool(((dbeta - want[0]).abs() <= U * K * want[1]).all()), "dbeta"
    assert bool(((dgamma - want[2]).abs() <= U * K * want[3]).all()), "dgamma"
    for i in at.tolist():
        xh, dz, sxh, sdz = slopes(i, i + 1)
        b = int(member[i])

        def spread_out(v):
            return (v[b] / count[b]).repeat_interleave(c // groups)[None]
        rr = r[b].repeat_interleave(c // groups)[None]
        value = rr * (dz * g64 - spread_out(s1) - xh * spread_out(s2))
        size = rr * (sdz * g64.abs() + spread_out(a1) + sxh * spread_out(a2))
        assert bool(((dx[i:i + 1].double() - value).abs() <= U * K * size + (HALF_BF16 * value.abs() if bf16 else 0)).all()), ("dx", i)
    assert not any(bool(torch.isnan(dx[a:b]).any()) for a, b in spans)


def ragged(n, samples):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(samples)
    share = torch.rand(samples, device=DEV, generator=gen, dtype=torch.float64)
    share[::31] = 0  # graphs without vertices
    ptr = torch.zeros(samples + 1, device=DEV, dtype=torch.int64)
    ptr[1:] = (torch.cumsum(share, 0) / share.sum() * n).round().long()
    ptr[-1] = n
    return ptr


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,c,groups", [(560_003, 256, 32), (1_000_003, 140, 7), (110_003, 1400, 1)])
def test_beyond_the_caches(n, c, groups, dtype):
    """Just above 256 MB: whole, in many samples, by row."""
    assert (1 << 28) < n * c * dtype.itemsize < (1 << 30)
    check(n, c, groups, dtype, "silu")
    check(n, c, groups, dtype, "none", samples=700, ptr=ragged(n, 700))
    check(n, c, 1, dtype, "silu", samples=n)


@pytest.mark.parametrize("n,c,groups", [(2_200_003, 128, 16), (180_003, 1500, 1)])
def test_in_many_tiles(n, c, groups):
    """2^28 values and more: 2,048 tiles of 256 threads."""
    assert n * c > 1 << 28
    check(n, c, groups, torch.float32, "silu")
    check(n, c, groups, torch.float32, "none", samples=3000, ptr=ragged(n, 3000))


def test_offsets_beyond_31_bits():
    n, c = 17_000_003, 128
    assert n * c > 1 << 31
    check(n, c, 16, torch.bfloat16, "silu")
    check(n, c, 16, torch.bfloat16, "none", samples=50_000, ptr=ragged(n, 50_000))
    check(n, c, 1, torch.bfloat16, "silu", samples=n)


@pytest.mark.parametrize("n,c,groups,dtype", [(20_003, 1024, 1, torch.float32), (300_001, 64, 1, torch.float32), (300_001, 64, 4, torch.bfloat16), (70_007, 602, 1, torch.bfloat16),
                                              (1_500_001, 8, 1, torch.float32)])
def test_rows_by_themselves_that_workgroups_walk_over(n, c, groups, dtype):
    check(n, c, groups, dtype, "silu", samples=n)


@pytest.mark.parametrize("c,groups,dtype", [(100, 10, torch.float32), (128, 16, torch.bfloat16)])
def test_small_samples_that_workgroups_walk_over(c, groups, dtype):
    """More samples than column sums are kept for."""
    n, samples = 200_003, 9000
    ptr = ragged(n, samples)
    check(n, c, groups, dtype, "silu", samples=samples, ptr=ptr, hint=int((ptr[1:] - ptr[:-1]).max()))
    check(n, c, groups, dtype, "none", samples=samples, ptr=ptr, hint=3)
