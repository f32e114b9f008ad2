"""Training a part of the vertices at a time: rows looked up by id and their table's gradient, hidden rows kept in 8 bits, layers, norm, loss, AdamW
and Muon together, against automatic differentiation of the same step in 64 bits on the host."""
import importlib.util
import os

import pytest
import torch

import paper_2104_06700_amd as gnn
import synth
from test_gpu_muon import allowed, newton_schulz

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32

_spec = importlib.util.spec_from_file_location("train_sage_parts", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                                                                               "train_sage_parts.py"))
train_sage_parts = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(train_sage_parts)
WIDTHS = (20, 48, 40, 7)


def trainer(count=3, **kw):
    el = synth.make_graph("rmat_sparse_stack", scale=0.0003, seed=11)
    x = synth.normal_features(el.n, WIDTHS[0], 1).to(DEV)
    labels = torch.randint(-3, WIDTHS[-1], (el.n,), generator=torch.Generator().manual_seed(2)).clamp(min=-1).to(torch.int32).to(DEV)
    parts = train_sage_parts.cut(el.dst.to(DEV), el.src.to(DEV), el.n, labels, count)
    return el, train_sage_parts.PartTrainer(parts, x, labels, WIDTHS, groups=4, lr=1e-2, weight_decay=0.1, **kw)


def held(t, p, dtype=torch.float64):
    """The hidden rows of the vertices outside p, as they are kept now."""
    rows = []
    for l in t.layers[:-1]:
        y = torch.empty(p.n - p.own, l["w"].shape[1], device=DEV)
        gnn.gnn_load_rows(l["store"], y, p.ids[p.own:])
        rows.append(y.to(dtype).cpu())
    return rows


def reference(el, t, p, table, weights, outside):
    """Loss, gradients (table first) and hidden rows of a step, in 64 bits, from the edges of the whole graph."""
    ids = p.ids.long().cpu()
    a = torch.zeros(el.n, el.n, dtype=torch.float64)
    a.index_put_((el.dst.long(), el.src.long()), torch.ones(el.e, dtype=torch.float64), accumulate=True)
    a = a[ids[:p.own]]
    degree = a.sum(1, keepdim=True)
    a = a[:, ids]
    assert torch.equal(a.sum(1, keepdim=True), degree)  # no edge is missing
    a[:, :p.own] += torch.eye(p.own, dtype=torch.float64)
    a /= degree + 1
    table = table.clone().requires_grad_()
    ps = [q.clone().requires_grad_() for q in weights]
    it = iter(ps)
    x, hidden = table[ids], []
    for i, l in enumerate(t.layers):
        w, b = next(it), next(it)
        x = a @ x @ w + b
        if not l["last"]:
            gamma, beta = next(it), next(it)
            v = x.view(p.own, t.groups, -1)
            mean = v.mean((0, 2), keepdim=True)
            var = ((v - mean) ** 2).mean((0, 2), keepdim=True)
            x = torch.relu(((v - mean) / torch.sqrt(var + 1e-5)).view(p.own, -1) * gamma + beta)
            hidden.append(x.detach())
            x = torch.cat([x, outside[i]])
    labels = p.labels[:p.own].long().cpu()
    there = labels >= 0
    loss = -torch.log_softmax(x, 1)[there].gather(1, labels[there][:, None]).mean()
    loss.backward()
    return float(loss.detach()), [table.grad] + [q.grad for q in ps], hidden


@pytest.mark.parametrize("count", [3, 1])
def test_a_step_of_a_part(count):
    el, t = trainer(count, embedding=True, muon=True)
    for p in t.parts:  # every vertex has hidden rows that a step left
        t.step(p)
    p = t.parts[count // 2]
    for m in t.momentum:
        m.zero_()
    start = [q.double().cpu() for q in t.params]
    outside = held(t, p)
    assert count == 1 or float(outside[0].abs().max()) > 0
    t.step(p)
    torch.cuda.synchronize()
    loss, grads, hidden = reference(el, t, p, start[0], start[1:], outside)
    # as for the whole graph: sums of some hundred fp32 terms through three layers, and gates next to zero that may stand the other way
    assert abs(float(t.loss) - loss) <= 1e-5 * abs(loss)
    assert len(t.grads) == len(grads) and t.grads[0] is t.dtable
    for g, want in zip(t.grads, grads):
        off = float((g.double().cpu() - want).norm() / want.norm())
        assert off <= 1e-4, (tuple(g.shape), off)
    left_out = torch.ones(el.n, dtype=torch.bool)
    left_out[p.ids.long().cpu()] = False
    assert (count == 1) == (not bool(left_out.any())) and float(t.dtable.cpu()[left_out].abs().sum()) == 0.0
    # the hidden rows of the part are kept: each within 2^-4 of itself, or half the least step of its block, 2^-10 of at most 2 / 448 of the largest
    for l, want in zip(t.layers, hidden):
        got = torch.empty(p.own, want.shape[1], device=DEV)
        gnn.gnn_load_rows(l["store"], got, p.ids[:p.own])
        blocks = [want[:, c:c + gnn.GNN_STORE_BLOCK].abs().amax(1, keepdim=True).expand(-1, want[:, c:c + gnn.GNN_STORE_BLOCK].shape[1])
                  for c in range(0, want.shape[1], gnn.GNN_STORE_BLOCK)]
        top = torch.cat(blocks, 1)
        assert ((got.double().cpu() - want).abs() <= 2.0 ** -4 * want.abs() + (2.0 ** -10 / 224 + 1e-4) * top).all()
    # weights by Muon, from the gradients as they are and no momentum before; the rest by AdamW
    for l, m in zip(t.layers, t.momentum):
        k = next(i for i, q in enumerate(t.params) if q is l["w"])
        g = l["dw"].double().cpu()
        assert torch.equal(m, l["dw"])
        o = newton_schulz(g * 1.95)
        scale = max(1.0, g.shape[1] / g.shape[0]) ** 0.5
        want = start[k] * (1 - t.muon_lr * 0.1) - t.muon_lr * scale * o
        far = float((l["w"].double().cpu() - want).norm())
        assert far <= t.muon_lr * scale * 2 * allowed(F32, o) + 4.1 * 2.0 ** -24 * float(want.norm())


def test_a_captured_step_repeats_itself():
    """Forward, backward and the update of the weights in one graph, from the same state each time."""
    _, t = trainer(embedding=True, muon=True)
    for p in t.parts:
        t.step(p)
    p = t.parts[1]
    state = t.params + t.momentum + [l["store"] for l in t.layers[:-1]]
    start = [s.clone() for s in state]

    def restore():
        for s, q in zip(state, start):
            s.copy_(q)

    def run():
        t.forward(p)
        t.backward(p)
        gnn.gnn_muon_step(t.muon, t.muon_lr, workspace=t.workspace)
    run()
    torch.cuda.synchronize()
    want = [s.clone() for s in state + t.grads + [t.loss]]
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        restore()
        for g in t.grads + [t.loss]:
            g.fill_(float("nan"))
        t.workspace.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, state + t.grads + [t.loss]))


@pytest.mark.parametrize("kw", [{}, dict(embedding=True, state_bits=8), dict(muon=True), dict(embedding=True, muon=True, state_bits=8)])
def test_some_epochs(kw):
    _, t = trainer(4, **kw)
    before = [q.clone() for q in t.params]
    for _ in range(3):
        for p in t.parts:
            loss = t.step(p)
    assert bool(torch.isfinite(loss).all()) and all(bool(torch.isfinite(q).all()) for q in t.params)
    assert all(not torch.equal(q, b) for q, b in zip(t.params, before))


def test_one_graph_with_weights_by_muon():
    """The whole graph at a time: the same gradients with either optimizer, and the weights moved by orthogonal updates."""
    kw = dict(scale=0.002, widths=(100, 64, 16), labelled=0.5)
    a, b = train_sage_parts.train_sage.make(muon=True, **kw), train_sage_parts.train_sage.make(**kw)
    start = [l["w"].double().cpu() for l in a.layers]
    a.step(), b.step()
    torch.cuda.synchronize()
    assert torch.equal(a.loss, b.loss) and all(torch.equal(p, q) for p, q in zip(a.grads, b.grads))
    for p, q, r in zip(a.params, b.params, a.grads):
        if not any(p is l["w"] for l in a.layers):
            assert torch.equal(p, q)
    for l, w0 in zip(a.layers, start):
        o = newton_schulz(l["dw"].double().cpu() * 1.95)
        scale = max(1.0, o.shape[1] / o.shape[0]) ** 0.5
        want = w0 * (1 - a.muon_lr * 1e-2) - a.muon_lr * scale * o
        far = float((l["w"].double().cpu() - want).norm())
        assert far <= a.muon_lr * scale * 2 * allowed(F32, o) + 4.1 * 2.0 ** -24 * float(want.norm())
