"""Newton-Schulz products and the optimizer step that uses them, against the formulas in 64 bits."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
COEFFICIENTS = gnn.GNN_NEWTON_SCHULZ


def newton_schulz(u, steps=5, eps=1e-7, coefficients=COEFFICIENTS):
    """O from the definition, in 64 bits."""
    a, b, c = coefficients
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        m = x @ x.t()
        x = a * x + (b * m + c * (m @ m)) @ x
    return x.t() if tall else x


# How far from it products in fp32 may take the result, in 2-norms.  The roundings of a product are of either sign: an error of about 2^-24 of what is
# summed, as large as |X| at the start, 1.  A direction of small singular values grows by 3.4445 a step, 485 in five, and errors in it with it; near 1,
# where the slope is about 1, the errors of a step are some ten times 2^-24 sqrt(m) of |X|, less than that up to m = 2,600.  Four times all
# that.  bf16 matrices: operands of 16 bits, each off by 2^-18.
def allowed(dtype, want):
    unit = 2.0 ** -24 if dtype == F32 else 2.0 ** -18
    half = 2.0 ** -24 if dtype == F32 else 2.0 ** -8  # the result's own rounding
    return 4 * 485 * unit * max(1.0, float(want.norm())) + half * float(want.norm())


def matrix(rows, cols, dtype, gen, kind="normal"):
    x = torch.randn(rows, cols, generator=gen)
    if kind == "decaying":
        k = min(rows, cols)
        x = (torch.randn(rows, k, generator=gen) * torch.exp2(-10 * torch.rand(k, generator=gen))) @ torch.randn(k, cols, generator=gen)
    elif kind == "rank one":
        x = torch.randn(rows, 1, generator=gen) @ torch.randn(1, cols, generator=gen)
    return x.to(dtype).to(DEV)


def orthogonalize(ins, outs=None, **kw):
    outs = [torch.full_like(u, float("nan")) for u in ins] if outs is None else outs
    t = gnn.OrthogonalizeTensors(ins, outs)
    ws = torch.full((max(1, gnn.gnn_orthogonalize_workspace_bytes(t)),), 255, device=DEV, dtype=torch.uint8)
    gnn.gnn_orthogonalize(t, workspace=ws, **kw)
    return outs


def check(o, u, **kw):
    want = newton_schulz(u, **kw)
    assert torch.isfinite(o).all()
    far = float((o.double() - want).norm())
    assert far <= allowed(u.dtype, want), (far, float(want.norm()))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (9, 1), (2, 2), (16, 31), (33, 32), (47, 256), (100, 256), (256, 256), (602, 16), (65, 513), (520, 300), (1000, 130), (1100, 1300), (2049, 2100)])
def test_one_matrix(rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 1000 + cols)
    u = matrix(rows, cols, dtype, gen)
    check(orthogonalize([u])[0], u)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["decaying", "rank one"])
@pytest.mark.parametrize("rows,cols", [(64, 200), (300, 100), (600, 520)])
def test_matrices_of_small_singular_values(rows, cols, kind, dtype):
    gen = torch.Generator().manual_seed(rows)
    u = matrix(rows, cols, dtype, gen, kind)
    check(orthogonalize([u])[0], u)


@pytest.mark.parametrize("factor", [1e-30, 1e30, 3e-42])
def test_the_size_of_a_matrix_does_not_matter(factor):
    """Squares of its values neither overflow nor vanish; eps is what a tiny matrix is divided by."""
    u = matrix(40, 90, F32, torch.Generator().manual_seed(1)) * factor
    eps = 1e-7 if factor > 1 else 1e-60
    check(orthogonalize([u], eps=eps)[0], u, eps=eps)


def test_zero_and_not_finite_matrices_stay_by_themselves():
    gen = torch.Generator().manual_seed(2)
    ins = [matrix(50, 70, F32, gen) for _ in range(4)]
    ins[1].zero_()
    ins[2][3, 4] = float("nan")
    ins[3][49, 69] = -float("inf")
    outs = orthogonalize(ins)
    check(outs[0], ins[0])
    assert (outs[1] == 0).all() and torch.isnan(outs[2]).all() and torch.isnan(outs[3]).all()


def test_many_matrices_of_all_kinds_at_once():
    gen = torch.Generator().manual_seed(3)
    shapes = [(5, 9), (100, 256), (700, 600), (256, 47), (1, 3), (600, 530), (2, 2)] * 6 + [(0, 5), (5, 0)]
    ins = [matrix(r, c, BF16 if k % 3 == 0 else F32, gen) for k, (r, c) in enumerate(shapes)]
    outs = orthogonalize(ins)
    for k, (u, o) in enumerate(zip(ins, outs)):
        if u.numel():
            alone = orthogonalize([u])[0]
            assert torch.equal(o, alone), k  # others in the call change nothing
    for k in (0, 1, 2, 3, 5):
        check(outs[k], ins[k])


@pytest.mark.parametrize("rows,cols", [(30, 45), (45, 30), (520, 600)])
def test_strides_and_in_place(rows, cols):
    gen = torch.Generator().manual_seed(4)
    wide = torch.randn(rows, cols + 13, generator=gen).to(DEV)
    u = wide[:, 3:3 + cols]
    want = orthogonalize([u.contiguous()])[0]
    out = torch.full((rows, cols + 5), float("nan"), device=DEV)
    orthogonalize([u], [out[:, :cols]])
    assert torch.equal(out[:, :cols], want) and torch.isnan(out[:, cols:]).all()
    left = wide.clone()
    orthogonalize([u], [u])
    assert torch.equal(u, want) and torch.equal(wide[:, :3], left[:, :3]) and torch.equal(wide[:, 3 + cols:], left[:, 3 + cols:])


@pytest.mark.parametrize("steps,coefficients", [(1, COEFFICIENTS), (2, (1.5, -0.5, 0.0)), (12, (1.5, -0.5, 0.0)), (8, (2.0, -1.5, 0.5))])
def test_other_steps_and_coefficients(steps, coefficients):
    u = matrix(60, 100, F32, torch.Generator().manual_seed(5))
    o = orthogonalize([u], steps=steps, coefficients=coefficients)[0]
    check(o, u, steps=steps, coefficients=coefficients)
    if steps == 12:  # converged: orthogonal rows
        assert float((o @ o.t() - torch.eye(60, device=DEV)).abs().max()) < 1e-4


def make_step(shapes, dtype, master, gen):
    ps = [torch.randn(r, c, generator=gen) * 0.1 for r, c in shapes]
    masters = [p.clone().to(DEV) for p in ps] if master else None
    ps = [p.to(dtype).to(DEV) for p in ps]
    gs = [(torch.randn(r, c, generator=gen) * 1e-3).to(dtype).to(DEV) for r, c in shapes]
    ms = [(torch.randn(r, c, generator=gen) * 1e-3).to(DEV) for r, c in shapes]
    return ps, gs, ms, masters


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype,master", [(F32, False), (BF16, False), (BF16, True)])
def test_a_step(dtype, master, nesterov):
    gen = torch.Generator().manual_seed(6)
    shapes = [(100, 256), (256, 256), (256, 47), (602, 16), (530, 700)]
    ps, gs, ms, masters = make_step(shapes, dtype, master, gen)
    gs[3] = None
    lr, mu, decay, gs_factor = 0.02, 0.9, 0.1, 0.5
    start = [(p.cpu().double() if masters is None else q.cpu().double(), m.cpu().double()) for p, m, q in zip(ps, ms, masters or ps)]
    t = gnn.MuonTensors(ps, gs, ms, masters, weight_decay=decay)
    ws = torch.empty(gnn.gnn_muon_workspace_bytes(t), device=DEV, dtype=torch.uint8)
    left = ps[3].clone(), ms[3].clone()
    gnn.gnn_muon_step(t, lr, momentum=mu, nesterov=nesterov, grad_scale=torch.full((1,), gs_factor, device=DEV), workspace=ws)
    assert torch.equal(ps[3], left[0]) and torch.equal(ms[3], left[1])
    for k, (r, c) in enumerate(shapes):
        if gs[k] is None:
            continue
        p0, m0 = start[k]
        g = gs[k].cpu().double() * gs_factor
        m = mu * m0 + g
        # momentum itself, both products and the sum are rounded: four halves of a step, of terms that may cancel
        assert ((ms[k].cpu().double() - m).abs() <= 4.1 * 2.0 ** -24 * (mu * m0.abs() + g.abs())).all()
        u = g + mu * m if nesterov else m
        o = newton_schulz(u)
        # U is made of fp32 numbers, a few roundings off, which grow like those of the products
        off = 2 * (allowed(dtype, o) - (2.0 ** -8 * float(o.norm()) if dtype == BF16 else 0.0))
        scale = max(1.0, c / r) ** 0.5
        want = p0 * (1 - lr * decay) - lr * scale * o
        for got, half in ((ps[k], 2.0 ** -24 if dtype == F32 else 2.0 ** -8), (masters[k] if masters else None, 2.0 ** -24)):
            if got is None:
                continue
            far = float((got.cpu().double() - want).norm())
            assert far <= lr * scale * off + (3 * 2.0 ** -24 + half) * float(want.norm()) * 1.01


def test_gradients_that_are_not_finite_and_set_grads():
    gen = torch.Generator().manual_seed(7)
    shapes = [(20, 30), (40, 10)]
    ps, gs, ms, _ = make_step(shapes, F32, False, gen)
    t = gnn.MuonTensors(ps, [None, None], ms)
    assert gnn.gnn_muon_workspace_bytes(t) == 0
    before = [p.clone() for p in ps]
    gnn.gnn_muon_step(t, 0.1)
    assert all(torch.equal(p, q) for p, q in zip(ps, before))
    gs[1][0, 0] = float("inf")
    t.set_grads(gs)
    ws = torch.empty(gnn.gnn_muon_workspace_bytes(t), device=DEV, dtype=torch.uint8)
    gnn.gnn_muon_step(t, 0.1, workspace=ws)
    assert torch.isfinite(ps[0]).all() and not torch.equal(ps[0], before[0]) and torch.isnan(ps[1]).all()


@pytest.mark.parametrize("shapes", [[(100, 256), (256, 256), (256, 47)], [(600, 700)]])
def test_replays_and_other_streams(shapes):
    gen = torch.Generator().manual_seed(8)
    ps, gs, ms, _ = make_step(shapes, F32, False, gen)
    start = [x.clone() for x in ps + ms]
    t = gnn.MuonTensors(ps, gs, ms, weight_decay=0.01)
    ws = torch.empty(gnn.gnn_muon_workspace_bytes(t), device=DEV, dtype=torch.uint8)

    def reset():
        for x, s in zip(ps + ms, start):
            x.copy_(s)
        ws.fill_(255)
        torch.cuda.synchronize()
    gnn.gnn_muon_step(t, 0.02, workspace=ws)
    gnn.gnn_muon_step(t, 0.02, workspace=ws)
    torch.cuda.synchronize()
    want = [x.clone() for x in ps + ms]
    side = torch.cuda.Stream()
    reset()
    for _ in range(2):
        gnn.gnn_muon_step(t, 0.02, workspace=ws, stream=side)
    side.synchronize()
    assert all(torch.equal(x, w) for x, w in zip(ps + ms, want))
    graph = torch.cuda.CUDAGraph()
    reset()
    with torch.cuda.graph(graph):
        gnn.gnn_muon_step(t, 0.02, workspace=ws)
    for _ in range(2):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, w) for x, w in zip(ps + ms, want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(60, 100), (1100, 1000), (2049, 2100)])
@pytest.mark.parametrize("coefficients", [(8.0, -2.0, 0.5), (0.5, 0.2, 0.1), (3.0, 4.0, 0.0), (2.0, 0.0, 0.0)])
def test_coefficients_that_let_singular_values_grow_or_vanish(coefficients, rows, cols, dtype):
    steps = 3
    a, b, c = (abs(x) for x in coefficients)
    u = matrix(rows, cols, dtype, torch.Generator().manual_seed(9))
    o = orthogonalize([u], steps=steps, coefficients=coefficients)[0]
    # A step's products are off by some ten times 2^-24 sqrt(m) (operands of 23 bits at least: twice that) of what they sum, whose size the same polynomial with
    # positive coefficients bounds; later steps take an error by at most the largest slope of the polynomial between 0 and the largest singular value.
    x = u.double()
    x = x / (x.norm() + 1e-7)
    far, m = 2.0 ** -23 * float(x.norm()), min(rows, cols)
    for _ in range(steps):
        top = float(torch.linalg.matrix_norm(x, 2))
        terms, slope = a + b * top ** 2 + c * top ** 4, a + 3 * b * top ** 2 + 5 * c * top ** 4
        far = far * slope + 20 * 2.0 ** -24 * m ** 0.5 * terms * float(x.norm())
        x = newton_schulz_step(x, coefficients)
    half = 2.0 ** -24 if dtype == F32 else 2.0 ** -8
    assert torch.isfinite(o).all()
    assert float((o.double() - x).norm()) <= far + half * float(x.norm())


def newton_schulz_step(x, coefficients):
    a, b, c = coefficients
    if x.shape[0] > x.shape[1]:
        return newton_schulz_step(x.t(), coefficients).t()
    m = x @ x.t()
    return a * x + (b * m + c * (m @ m)) @ x


@pytest.mark.parametrize("steps", [1, 5, 9])
@pytest.mark.parametrize("rows,cols", [(40, 90), (300, 200), (1100, 1000)])
@pytest.mark.parametrize("factor", [1e-3, 1e-10, 1e-14, 1e-20, 1e-28])
def test_matrices_far_smaller_than_eps(factor, rows, cols, steps):
    """X is as small then, and the result is as close to it as that of a large one, relative to its size."""
    u = matrix(rows, cols, F32, torch.Generator().manual_seed(10)) * factor
    eps = 1e-7
    o = orthogonalize([u], steps=steps, eps=eps)[0]
    want = newton_schulz(u, steps=steps, eps=eps)
    # while X is small a step multiplies it by 3.4445, its errors with it; near 1 as in allowed()
    grows = min(3.4445 ** steps, max(1.0, float(want.norm())) * 485 / float((u.double() / (u.double().norm() + eps)).norm()))
    start = float((u.double() / (u.double().norm() + eps)).norm())
    assert torch.isfinite(o).all()
    assert float((o.double() - want).norm()) <= 4 * 2.0 ** -24 * grows * start + steps * 20 * 2.0 ** -24 * min(rows, cols) ** 0.5 * float(want.norm())


@pytest.mark.parametrize("coefficients", [COEFFICIENTS, (3.0, 4.0, 0.0)])
@pytest.mark.parametrize("eps", [1e-300, 5e-324, 1e300])
def test_zeros_with_any_eps(eps, coefficients):
    assert (orthogonalize([torch.zeros(40, 50, device=DEV)], eps=eps, coefficients=coefficients)[0] == 0).all()
