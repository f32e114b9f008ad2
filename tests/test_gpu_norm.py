"""Group norm with activation, channels last, and its gradients against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2104_06700_amd as gnn

DEV = "cuda:0"
ACTS = {"none": gnn.GNN_ACT_NONE, "relu": gnn.GNN_ACT_RELU, "silu": gnn.GNN_ACT_SILU}
# Rounding bounds.  U: one fp32 operation.  A statistic adds at most 16 values one after the other in fp32 at these sizes (a tile of 4096
# values on 256 threads) before wider sums take over, and about as many operations form a result: K operations each off by U, on
# magnitudes that the reference returns beside its values (`size`).  exp's argument is rounded too: |z| more operations.
U, K = 2.0 ** -23, 32
HALF_BF16 = 2.0 ** -8


def reference(x, gamma, beta, groups, ptr, act, eps, dy=None, stats=None):
    """Results and their magnitudes in 64 bits: {name: (value, size)}."""
    n, c = x.shape
    x, gamma, beta = (t.astype(np.float64) for t in (x, gamma, beta))
    b = len(ptr) - 1
    y, sy = np.zeros((n, c)), np.zeros((n, c))
    mean, rstd = np.zeros((b, groups)), np.full((b, groups), 1 / math.sqrt(eps))
    smean, srstd = np.zeros((b, groups)), rstd.copy()
    dx, sdx = np.zeros((n, c)), np.zeros((n, c))
    dgamma, dbeta, sdgamma, sdbeta = (np.zeros(c) for _ in range(4))
    k = c // groups
    gm, bt = gamma.reshape(groups, k), beta.reshape(groups, k)
    for s in range(b):
        lo, hi = ptr[s], ptr[s + 1]
        if hi == lo:
            continue
        xs = x[lo:hi].reshape(hi - lo, groups, k)
        m = xs.mean((0, 2))
        var = ((xs - m[:, None]) ** 2).mean((0, 2))
        r = 1 / np.sqrt(var + eps)
        mean[s], rstd[s] = m, r
        smean[s], srstd[s] = np.abs(xs).mean((0, 2)), r * (1 + np.abs(m) * r * U)
        if stats is not None:  # what the backward pass is given
            m, r = stats[0][s].astype(np.float64), stats[1][s].astype(np.float64)
        xh = (xs - m[:, None]) * r[:, None]
        sxh = np.abs(xh) + np.abs(m[:, None] * r[:, None]) + 1
        z = xh * gm + bt
        sz = sxh * np.abs(gm) + np.abs(bt)
        sig = 1 / (1 + np.exp(-z))
        if act == "relu":
            out, slope, rough = np.maximum(z, 0), (z > 0).astype(float), np.zeros_like(z)
        elif act == "silu":
            out, slope, rough = z * sig, sig * (1 + z * (1 - sig)), np.ones_like(z)
        else:
            out, slope, rough = z, np.ones_like(z), np.zeros_like(z)
        y[lo:hi] = out.reshape(-1, c)
        sy[lo:hi] = (1.1 * sz + rough * np.abs(out) * np.abs(z)).reshape(-1, c)
        if dy is None:
            continue
        d = dy[lo:hi].astype(np.float64).reshape(hi - lo, groups, k)
        dz = d * slope
        sdz = np.abs(dz) + rough * np.abs(d) * (sz + np.abs(z))  # the slope of silu changes by at most 0.5 sz
        s1, s2 = (dz * gm).mean((0, 2)), (dz * gm * xh).mean((0, 2))
        a1, a2 = (sdz * np.abs(gm)).mean((0, 2)), (sdz * np.abs(gm) * sxh).mean((0, 2))
        dx[lo:hi] = (r[:, None] * (dz * gm - s1[:, None] - xh * s2[:, None])).reshape(-1, c)
        sdx[lo:hi] = (r[:, None] * (sdz * np.abs(gm) + a1[:, None] + sxh * a2[:, None])).reshape(-1, c)
        dbeta += dz.sum(0).reshape(-1)
        dgamma += (dz * xh).sum(0).reshape(-1)
        sdbeta += sdz.sum(0).reshape(-1)
        sdgamma += (sdz * sxh).sum(0).reshape(-1)
    return dict(y=(y, sy), mean=(mean, smean), rstd=(rstd, srstd), dx=(dx, sdx), dgamma=(dgamma, sdgamma), dbeta=(dbeta, sdbeta))


def close(got, want, what, bf16=False):
    value, size = want
    g = got.detach().float().cpu().numpy().astype(np.float64)
    assert g.shape == value.shape, (what, g.shape, value.shape)
    assert np.isfinite(g).all(), f"{what}: not finite"
    bound = U * K * size + (HALF_BF16 * np.abs(value) if bf16 else 0) + 1e-37
    err = np.abs(g - value)
    if (err > bound).any():
        i = np.unravel_index(np.argmax(err - bound), err.shape)
        raise AssertionError(f"{what}: {(err > bound).sum()} of {err.size} off; worst at {i}: {g[i]!r}, expected {value[i]!r}, bound {bound[i]:.3e}")


def inputs(n, c, seed, dtype=torch.float32, offset=1.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy((rng.normal(size=(n, c)) * (0.5 + rng.random(c)) + offset * rng.normal(size=c)).astype(np.float32)).to(dtype)
    dy = torch.from_numpy(rng.normal(size=(n, c)).astype(np.float32)).to(dtype)
    gamma = torch.from_numpy((1 + 0.2 * rng.normal(size=c)).astype(np.float32))
    beta = torch.from_numpy((0.3 * rng.normal(size=c)).astype(np.float32))
    return x, dy, gamma, beta


def on_device(t, ld=None, front=0):
    """The matrix on the device with row stride ld, `front` elements into a buffer that is otherwise NaN; matrix and buffer."""
    n, c = t.shape
    ld = ld or c
    buf = torch.full((front + n * ld + 16,), float("nan"), dtype=t.dtype, device=DEV)
    m = torch.as_strided(buf, (n, c), (ld, 1), front)
    m.copy_(t)
    return m, buf


def untouched(m, buf):
    """Nothing but the matrix has been written into its buffer."""
    inside = torch.zeros(buf.shape, dtype=torch.bool, device=DEV)
    torch.as_strided(inside, m.shape, m.stride(), m.storage_offset()).fill_(True)
    return bool(torch.isnan(buf[~inside].float()).all())


def check(n, c, groups, ptr, act, dtype=torch.float32, seed=0, eps=1e-5, hint=0, uniform=0, lds=(None, None, None), front=0, ptr_dtype=torch.int64,
          affine=True, offset=1.0):
    bf16 = dtype == torch.bfloat16
    x, dy, gamma, beta = inputs(n, c, seed, dtype, offset)
    if act == "relu":  # the gate is open or shut beyond doubt: results next to zero are pushed away from it
        ref = reference(x.float().numpy(), gamma.numpy(), beta.numpy(), groups, ptr, "none", eps)["y"]
        x = torch.where(torch.from_numpy(np.abs(ref[0]) < 1e-3), x + (0.05 if not bf16 else 0.25), x)
    if not affine:
        gamma, beta = torch.ones(c), torch.zeros(c)
    b = len(ptr) - 1
    xd, _ = on_device(x, lds[0], front)
    y, ybuf = on_device(torch.full_like(x, float("nan")), lds[1], front)
    mean, rstd = torch.full((b, groups), float("nan"), device=DEV), torch.full((b, groups), float("nan"), device=DEV)
    g, be = (gamma.to(DEV), beta.to(DEV)) if affine else (None, None)
    kw = dict(act=ACTS[act], max_sample_rows=hint)
    if uniform:
        kw["n_samples"] = b
    else:
        kw["sample_ptr"] = torch.tensor(ptr, dtype=ptr_dtype, device=DEV)
    ws = torch.full((max(1, gnn.gnn_group_norm_workspace_bytes(n, c, groups, b, True)) // 4 + 1,), float("nan"), device=DEV)
    gnn.gnn_group_norm_fwd(xd, g, be, y, mean, rstd, groups, eps=eps, workspace=ws, **kw)
    torch.cuda.synchronize()
    ref = reference(x.float().numpy(), gamma.numpy(), beta.numpy(), groups, ptr, act, eps)
    where = f"n={n} c={c} groups={groups} samples={b} {act} {dtype}"
    close(mean, ref["mean"], "mean " + where)
    close(rstd, ref["rstd"], "rstd " + where)
    close(y, ref["y"], "y " + where, bf16)
    assert untouched(y, ybuf), where
    # backward, from these statistics
    ref = reference(x.float().numpy(), gamma.numpy(), beta.numpy(), groups, ptr, act, eps, dy.float().numpy(),
                    (mean.cpu().numpy(), rstd.cpu().numpy()))
    dyd, _ = on_device(dy, lds[1], front)
    dx, dxbuf = on_device(torch.full_like(x, float("nan")), lds[2], front)
    dgamma, dbeta = torch.full((c,), float("nan"), device=DEV), torch.full((c,), float("nan"), device=DEV)
    ws.fill_(float("nan"))
    gnn.gnn_group_norm_bwd(xd, g, be, mean, rstd, dyd, dx, dgamma, dbeta, groups, workspace=ws, **kw)
    torch.cuda.synchronize()
    close(dbeta, ref["dbeta"], "dbeta " + where)
    close(dgamma, ref["dgamma"], "dgamma " + where)
    close(dx, ref["dx"], "dx " + where, bf16)
    assert untouched(dx, dxbuf), where
    # parts of the gradients give the same bits
    only = torch.empty_like(dgamma)
    gnn.gnn_group_norm_bwd(xd, g, be, mean, rstd, dyd, None, only, None, groups, workspace=ws, **kw)
    again = torch.empty_like(x.to(DEV))
    gnn.gnn_group_norm_bwd(xd, g, be, mean, rstd, dyd, again, None, None, groups, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert torch.equal(only, dgamma) and torch.equal(again, dx), where


@pytest.mark.gpu
@pytest.mark.parametrize("n,c,groups", [(1, 1, 1), (1, 64, 8), (2, 3, 3), (7, 5, 1), (300, 64, 8), (257, 100, 10), (1000, 37, 37), (513, 602, 14),
                                        (4096, 64, 8), (70, 1500, 3), (33, 4100, 4), (5, 2500, 2500), (2049, 9, 3), (3000, 256, 32)])
@pytest.mark.parametrize("act,dtype", [("none", torch.float32), ("relu", torch.float32), ("silu", torch.float32), ("silu", torch.bfloat16),
                                       ("relu", torch.bfloat16)])
def test_one_sample(n, c, groups, act, dtype):
    print("one sample", n, c, groups, act, dtype, flush=True)
    check(n, c, groups, [0, n], act, dtype, uniform=1)


@pytest.mark.gpu
@pytest.mark.parametrize("samples,rows", [(1000, 1), (333, 3), (64, 17), (40, 25), (7, 300), (2, 1500)])
@pytest.mark.parametrize("c,groups", [(64, 8), (100, 10), (37, 1), (6, 3), (250, 5)])
def test_samples_of_equal_size(samples, rows, c, groups):
    for act, dtype in (("silu", torch.float32), ("relu", torch.bfloat16)):
        print("equal samples", samples, rows, c, groups, act, dtype, flush=True)
        check(samples * rows, c, groups, list(range(0, samples * rows + 1, rows)), act, dtype, uniform=1)


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(3, 1), (4, 1), (8, 1), (9, 1), (64, 16), (129, 1), (192, 3), (256, 2), (256, 64), (300, 1), (512, 16), (602, 1), (770, 1),
                                      (1023, 1), (1024, 1), (1024, 128), (1025, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_vertex_by_itself(c, groups, dtype):
    for n, act in ((1, "silu"), (5, "none"), (1003, "silu"), (258, "relu")):
        print("rows", n, c, groups, dtype, act, flush=True)
        check(n, c, groups, list(range(n + 1)), act, dtype, uniform=1)
    check(77, c, groups, list(range(78)), "silu", dtype, uniform=1, lds=(c + 3, c + 1, c + 5), front=3, affine=False)


@pytest.mark.gpu
def test_small_samples_longer_than_registers_hold():
    """Many samples that one workgroup each reads again and again, narrow groups and a last vector that ends with the row among them."""
    rng = np.random.default_rng(7)
    for c, groups, most in ((128, 16, 250), (99, 9, 120), (35, 35, 700)):
        sizes = list(rng.integers(0, most, 260))
        ptr = [0] + [int(v) for v in np.cumsum(sizes)]
        for dtype in (torch.float32, torch.bfloat16):
            print("long", c, groups, most, dtype, flush=True)
            check(ptr[-1], c, groups, ptr, "silu", dtype, hint=most)


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups", [(1500, 3), (2000, 4), (2600, 2), (4096, 8), (4100, 5)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_wide_rows_in_many_small_samples(c, groups, dtype):
    for rows in (3, 9, 17):
        print("wide", rows, c, groups, dtype, flush=True)
        check(260 * rows, c, groups, list(range(0, 260 * rows + 1, rows)), "silu", dtype, uniform=1)


def ragged(name, rng):
    if name == "empty ones":
        sizes = [0, 0, 5, 0, 1, 130, 0, 64, 0, 0]
    elif name == "one giant":
        sizes = [1, 2, 3000, 0, 1, 4, 1]
    elif name == "ones":
        sizes = [1] * 700
    elif name == "tile borders":
        sizes = [64, 64, 63, 65, 128, 1, 127, 256, 0, 192]
    else:
        sizes = list(rng.integers(0, 51, 150))
    return [0] + [int(v) for v in np.cumsum(sizes)]


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["empty ones", "one giant", "ones", "tile borders", "many"])
@pytest.mark.parametrize("c,groups,dtype", [(64, 8, torch.float32), (100, 10, torch.float32), (47, 47, torch.bfloat16), (256, 1, torch.bfloat16), (3, 1, torch.float32)])
def test_ragged_samples(name, c, groups, dtype):
    ptr = ragged(name, np.random.default_rng(3))
    for hint, ptr_dtype, act in ((0, torch.int64, "silu"), (max(b - a for a, b in zip(ptr, ptr[1:])), torch.int32, "none"), (2, torch.int64, "relu")):
        print("ragged", name, c, groups, dtype, hint, flush=True)
        check(ptr[-1], c, groups, ptr, act, dtype, hint=hint, ptr_dtype=ptr_dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("c,groups,dtype", [(1000, 8, torch.float32), (1024, 1, torch.bfloat16), (1030, 5, torch.float32), (7, 1, torch.bfloat16), (512, 512, torch.float32)])
def test_samples_inside_and_across_tiles(c, groups, dtype):
    """Samples that begin and end with a tile, fill it, cross one border or several, and share one, beside samples without rows."""
    # a tile has 16384 values: 16 or 17 rows of the widest
    sizes = [16, 1, 15, 17, 16, 0, 3, 0, 13, 40, 8, 0, 0, 2, 1, 1, 33, 16, 100, 5, 0]
    ptr = [0] + [int(v) for v in np.cumsum(sizes)]
    for act, ptr_dtype in (("silu", torch.int64), ("relu", torch.int32)):
        print("tiles", c, groups, dtype, act, flush=True)
        check(ptr[-1], c, groups, ptr, act, dtype, ptr_dtype=ptr_dtype)
    # many more samples than tiles
    ptr = [0] + [int(v) for v in np.cumsum(np.random.default_rng(5).integers(0, 4, 400))]
    check(ptr[-1], c, groups, ptr, "silu", dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("lds,front", [((100, 104, 128), 0), ((101, 103, 107), 3), ((300, 100, 100), 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(lds, front, dtype):
    check(500, 100, 10, [0, 500], "silu", dtype, uniform=1, lds=lds, front=front)
    check(500, 100, 10, list(range(0, 501, 25)), "relu", dtype, uniform=1, lds=lds, front=front)


@pytest.mark.gpu
def test_without_affine_parameters_and_with_large_means():
    check(900, 64, 8, [0, 900], "none", uniform=1, affine=False)
    check(900, 64, 8, [0, 400, 900], "silu", affine=False)
    check(2000, 64, 8, [0, 2000], "none", uniform=1, offset=1e4)  # the mean is 10,000 times the deviation
    check(2000, 64, 8, list(range(0, 2001, 20)), "none", uniform=1, offset=1e4)


@pytest.mark.gpu
def test_constant_rows_have_no_deviation():
    for n, samples in ((640, 1), (640, 64)):
        x = torch.full((n, 32), 3.25, device=DEV)
        y = torch.empty_like(x)
        mean, rstd = torch.empty(samples, 4, device=DEV), torch.empty(samples, 4, device=DEV)
        beta = torch.arange(32, device=DEV, dtype=torch.float32)
        ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, 32, 4, samples), device=DEV, dtype=torch.uint8)
        gnn.gnn_group_norm_fwd(x, None, beta, y, mean, rstd, 4, n_samples=samples, workspace=ws, eps=1e-5)
        torch.cuda.synchronize()
        assert bool((mean == 3.25).all()) and torch.equal(y, beta.expand(n, 32))
        assert float((rstd * math.sqrt(1e-5) - 1).abs().max()) < 1e-6


@pytest.mark.gpu
def test_not_finite_values_stay_in_their_sample_and_group():
    n, c, groups, samples = 600, 64, 8, 6
    for hint_kw in (dict(n_samples=samples), dict(sample_ptr=torch.arange(0, n + 1, n // samples, device=DEV))):
        for bad in (float("nan"), float("inf")):
            x, dy, gamma, beta = (t.to(DEV) for t in inputs(n, c, 5))
            x[250, 17] = bad  # sample 2, group 2
            y = torch.empty_like(x)
            mean, rstd = torch.empty(samples, groups, device=DEV), torch.empty(samples, groups, device=DEV)
            ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, groups, samples, True), device=DEV, dtype=torch.uint8)
            gnn.gnn_group_norm_fwd(x, gamma, beta, y, mean, rstd, groups, act=gnn.GNN_ACT_RELU, workspace=ws, **hint_kw)
            torch.cuda.synchronize()
            hit = torch.zeros(samples, groups, dtype=torch.bool, device=DEV)
            hit[2, 2] = True
            assert torch.equal(torch.isnan(rstd), hit)
            rows = torch.zeros_like(x, dtype=torch.bool)
            rows[200:300, 16:24] = True
            assert torch.equal(torch.isnan(y), rows)


@pytest.mark.gpu
def test_other_streams_captures_and_repeats_give_the_same_bits():
    for n, c, groups, samples in ((5000, 100, 10, 1), (5000, 100, 10, 200)):
        x, dy, gamma, beta = (t.to(DEV) for t in inputs(n, c, 9))
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(samples, groups, device=DEV), torch.empty(samples, groups, device=DEV)
        dgamma, dbeta = torch.empty(c, device=DEV), torch.empty(c, device=DEV)
        ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, groups, samples, True), device=DEV, dtype=torch.uint8)

        def both(stream=None):
            gnn.gnn_group_norm_fwd(x, gamma, beta, y, mean, rstd, groups, n_samples=samples, act=gnn.GNN_ACT_SILU, workspace=ws, stream=stream)
            gnn.gnn_group_norm_bwd(x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, groups, n_samples=samples, act=gnn.GNN_ACT_SILU, workspace=ws,
                                   stream=stream)
        outs = (y, mean, rstd, dx, dgamma, dbeta)
        both()
        torch.cuda.synchronize()
        first = [t.clone() for t in outs]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        both(stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        for _ in range(3):
            for t in outs:
                t.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(first, outs))


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_against_differences_of_the_forward_call(act):
    """Directional derivatives of sum W Y: central differences over a step h are off by h^2 times the third derivative and by the
    rounding of Y, U K size |W| / h, added up over independent elements."""
    n, c, groups, ptr = 96, 24, 4, [0, 10, 10, 41, 96]
    x, w, gamma, beta = inputs(n, c, 21)
    b = len(ptr) - 1
    p = torch.tensor(ptr, device=DEV)
    ws = torch.empty(gnn.gnn_group_norm_workspace_bytes(n, c, groups, b, True), device=DEV, dtype=torch.uint8)
    mean, rstd = torch.empty(b, groups, device=DEV), torch.empty(b, groups, device=DEV)

    def f(x, gamma, beta):
        y = torch.empty(n, c, device=DEV)
        gnn.gnn_group_norm_fwd(x.to(DEV), gamma.to(DEV), beta.to(DEV), y, mean, rstd, groups, sample_ptr=p, act=ACTS[act], workspace=ws)
        return float((y.double().cpu() * w.double()).sum())
    f(x, gamma, beta)
    dx, dgamma, dbeta = torch.empty(n, c, device=DEV), torch.empty(c, device=DEV), torch.empty(c, device=DEV)
    gnn.gnn_group_norm_bwd(x.to(DEV), gamma.to(DEV), beta.to(DEV), mean, rstd, w.to(DEV), dx, dgamma, dbeta, groups, sample_ptr=p, act=ACTS[act], workspace=ws)
    rng = np.random.default_rng(4)
    size = reference(x.numpy(), gamma.numpy(), beta.numpy(), groups, ptr, act, 1e-5)["y"][1]
    h = 2.0 ** -7
    noise = U * K * float(np.sqrt(((size * np.abs(w.numpy())) ** 2).sum())) / h
    for which, grad in ((0, dx), (1, dgamma), (2, dbeta)):
        base = [x, gamma, beta]
        d = torch.from_numpy(rng.choice([-1.0, 1.0], size=base[which].shape).astype(np.float32))
        up, down = list(base), list(base)
        up[which], down[which] = base[which] + h * d, base[which] - h * d
        slope = (f(*up) - f(*down)) / (2 * h)
        want = float((grad.double().cpu() * d.double()).sum())
        curve = h * h * 4 * float(np.sqrt((grad.cpu().numpy().astype(np.float64) ** 2).sum()) + np.abs(w.numpy()).sum() / 4)
        assert abs(slope - want) <= noise + curve, (which, slope, want, noise, curve)


def test_reference_gradients_against_differences():
    """The reference itself, in 64 bits."""
    n, c, groups, ptr = 12, 6, 2, [0, 5, 5, 12]
    x, w, gamma, beta = (t.numpy().astype(np.float64) for t in inputs(n, c, 8))
    for act in ("none", "silu", "relu"):
        ref = reference(x, gamma, beta, groups, ptr, act, 1e-3, w)
        for which, name in enumerate(("dx", "dgamma", "dbeta")):
            base = [x, gamma, beta]
            for i in np.ndindex(base[which].shape):
                h = 1e-6
                f = []
                for step in (h, -h):
                    moved = [t.copy() for t in base]
                    moved[which][i] += step
                    f.append((reference(*moved, groups, ptr, act, 1e-3)["y"][0] * w).sum())
                assert abs((f[0] - f[1]) / (2 * h) - ref[name][0][i]) < 1e-6, (act, name, i)
