"""The statistics of the group norm where a row, a column or the mean is unlike the rest, against two passes in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2104_06700_amd as gnn

DEV = "cuda:0"
# U: one fp32 operation.  A statistic is a sum of terms of one sign (or of distances from the mean) of which at most some 32 are added one after the
# other, runs of four to 32 and then a tree, each off by U; the results take a handful of operations more.
U, K = 2.0 ** -23, 32


def forward(x, groups, ptr=None, samples=1, hint=0, gamma=None, beta=None, eps=1e-5):
    n, c = x.shape
    kw = dict(n_samples=samples)
    if ptr is not None:
        kw, samples = dict(sample_ptr=torch.tensor(ptr, device=DEV), max_sample_rows=hint), len(ptr) - 1
    xd = x.to(DEV)
    y = torch.full_like(xd, float("nan"))
    mean, rstd = (torch.full((samples, groups), float("nan"), device=DEV) for _ in range(2))
    ws = torch.full((gnn.gnn_group_norm_workspace_bytes(n, c, groups, samples) // 4 + 1,), float("nan"), device=DEV)
    gnn.gnn_group_norm_fwd(xd, None if gamma is None else gamma.to(DEV), None if beta is None else beta.to(DEV), y, mean, rstd, groups, eps=eps, workspace=ws, **kw)
    torch.cuda.synchronize()
    return [t.float().cpu().numpy().astype(np.float64) for t in (y, mean, rstd)]


def within(got, want, bound, what):
    err = np.abs(got - want)
    assert np.isfinite(got).all() and (err <= bound).all(), f"{what}: off by up to {np.max(err / bound):.3g} bounds"


def check(x, groups, what, ptr=None, samples=1, hint=0, eps=1e-5, rounded=True):
    n, c = x.shape
    bounds = ptr or [n // samples * i for i in range(samples + 1)]
    y, mean, rstd = forward(x, groups, ptr, samples, hint, eps=eps)
    for b, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        if lo == hi:
            continue
        v = x[lo:hi].double().numpy().reshape(hi - lo, groups, c // groups)
        m = v.mean((0, 2))
        d = v - m[None, :, None]
        m = m + d.mean((0, 2))
        d = v - m[None, :, None]
        r = 1 / np.sqrt((d ** 2).mean((0, 2)) + eps)
        where = f"{what}, sample {b}"
        within(rstd[b], r, U * K * r, "rstd, " + where)
        within(mean[b], m, U * np.abs(m) + U * K * np.abs(d).mean((0, 2)) + 1e-37, "mean, " + where)
        # rounded: the result may take the mean as it is stored
        xh = d * r[None, :, None]
        within(y[lo:hi].reshape(xh.shape), xh, U * K * (1 + np.abs(xh)) + rounded * U * (np.abs(m) * r)[None, :, None], "y, " + where)


def unlike(kind, n, c, seed):
    x = torch.from_numpy(np.random.default_rng(seed).normal(size=(n, c)).astype(np.float32))
    if kind == "zero":       # an isolated or a padding vertex in front of features of mean 30
        x += 30
        x[:1] = 0
    elif kind == "zero of 100":
        x += 100
        x[:1] = 0
    elif kind == "far":      # a hub
        x[:1] = 1000
    elif kind == "some far":
        x[:7] = 3000
    elif kind == "last far":
        x[-1:] = -1000
    return x


KINDS = ["zero", "zero of 100", "far", "some far", "last far"]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,c,groups", [(4096, 64, 8), (16384, 1, 1), (16384, 16, 4), (131072, 2, 2), (300000, 24, 24), (2000, 1500, 500)])
def test_one_sample_with_a_row_unlike_the_rest(kind, n, c, groups):
    print("one sample", kind, n, c, groups, flush=True)
    check(unlike(kind, n, c, n + c), groups, kind)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("c,groups", [(1, 1), (16, 4), (100, 10), (256, 1), (1030, 5)])
def test_samples_with_a_row_unlike_the_rest(kind, c, groups):
    """Every sample with a row of its own kind; nothing is known of their lengths."""
    sizes = [1, 1000, 17, 3000, 0, 2, 5000 if c < 500 else 50, 33]
    ptr = [0] + [int(v) for v in np.cumsum(sizes)]
    print("samples", kind, c, groups, flush=True)
    x = torch.cat([unlike(kind, n, c, 7 * n + c) for n in sizes])
    check(x, groups, kind, ptr)


@pytest.mark.gpu
@pytest.mark.parametrize("samples,rows", [(1, 1000), (6, 300)])
def test_a_column_unlike_the_rest_of_its_group(samples, rows):
    for at in (0, 999):
        x = unlike("none", samples * rows, 1000, at)
        x[:, at] += 1000
        check(x, 1, f"column {at}", samples=samples)


def paths(c, groups):
    """Ways through the kernels: (name, rows, arguments)."""
    yield "every vertex", 40, dict(samples=40)
    yield "a workgroup a sample", 300, dict(samples=12)
    yield "a workgroup a sample, longer than its registers", 12, dict(ptr=[0, 1, 1, 12], hint=1)
    yield "one sample", 5000, dict(samples=1)
    yield "tiles", 3000, dict(ptr=[0, 3, 3, 900, 901, 3000])


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(60, 1), (100, 1), (37, 1), (64, 8), (100, 10), (6, 3), (1200, 4)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_values_give_beta(c, groups, dtype):
    """The mean of equal values is that value and their deviation 0, whatever the value and their number."""
    beta = torch.linspace(-2, 3, c)
    for name, n, kw in paths(c, groups):
        for value in (1000.0, 1e4 + 1 / 3, -1e5, 3e-5):
            print("equal", name, c, groups, value, flush=True)
            x = torch.full((n, c), value).to(dtype)
            y, mean, rstd = forward(x, groups, beta=beta, **kw)
            rows = [n] if kw.get("samples") else [b - a for a, b in zip(kw["ptr"], kw["ptr"][1:])]
            there = np.array([r > 0 for r in rows]) if "ptr" in kw else slice(None)
            assert (mean[there] == float(x[0, 0])).all(), (name, value, mean)
            assert np.array_equal(y, np.broadcast_to(beta.to(dtype).double().numpy(), y.shape)), (name, value)
            # what is left of the squares is below the square of two units in the value's last place
            within(rstd, 1 / np.sqrt(1e-5) + 0 * rstd, (U + (2 * U * value) ** 2 / 1e-5 / 2 * U + 2 * U) / np.sqrt(1e-5) + 0 * rstd, "rstd " + name)


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(60, 1), (100, 1), (37, 1), (64, 8), (100, 10), (6, 3), (1200, 4)])
@pytest.mark.parametrize("mean,deviation", [(1e3, 0.1), (1e4, 1.0), (-1e5, 1.0)])
def test_a_mean_far_beyond_the_deviation(c, groups, mean, deviation):
    """The result is as close as that of the distances from the mean: its bound does not hold the mean."""
    for name, n, kw in paths(c, groups):
        print("large mean", name, c, groups, mean, deviation, flush=True)
        x = torch.from_numpy((mean + deviation * np.random.default_rng(n + c).normal(size=(n, c))).astype(np.float32))
        check(x, groups, name, rounded=False, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("c,groups", [(1, 1), (16, 4), (100, 10), (256, 1), (1030, 5)])
def test_a_row_unlike_the_rest_in_a_workgroup(kind, c, groups):
    """As above, one workgroup a sample: hints that are right or too small."""
    for sizes, hint in (([1, 17, 0, 2, 33, 10], 33), ([1, 1000, 17, 300, 0, 2], 1)):
        ptr = [0] + [int(v) for v in np.cumsum(sizes)]
        print("workgroups", kind, c, groups, hint, flush=True)
        check(torch.cat([unlike(kind, n, c, 5 * n + c) for n in sizes]), groups, kind, ptr, hint=hint)
