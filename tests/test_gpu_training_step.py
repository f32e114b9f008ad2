"""A whole training step of the library's calls (layers, group norm, loss, AdamW) against automatic differentiation of the same model in
64 bits on the host, and training with states in 32 and in 8 bits."""
import importlib.util
import os

import pytest
import torch

import paper_2104_06700_amd as gnn
import synth
from helpers import device_graph

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

_spec = importlib.util.spec_from_file_location("train_sage", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                                                                         "train_sage.py"))
train_sage = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(train_sage)


def reference(el, t, parameters):
    """Loss and gradients of the model, dense, in 64 bits."""
    n = el.n
    a = torch.zeros(n, n, dtype=torch.float64)
    a.index_put_((el.dst.long(), el.src.long()), torch.ones(el.e, dtype=torch.float64), accumulate=True)
    degree = a.sum(1, keepdim=True)
    a += torch.eye(n, dtype=torch.float64)
    a /= degree + 1
    ps = [p.clone().requires_grad_() for p in parameters]
    it = iter(ps)
    x = next(it)
    for l in t.layers:
        w, b = next(it), next(it)
        x = a @ x @ w + b
        if not l["last"]:
            gamma, beta = next(it), next(it)
            k = x.shape[1] // t.groups
            v = x.view(n, t.groups, k)
            mean = v.mean((0, 2), keepdim=True)
            var = ((v - mean) ** 2).mean((0, 2), keepdim=True)
            x = torch.relu(((v - mean) / torch.sqrt(var + 1e-5)).view(n, -1) * gamma + beta)
    labels = t.labels.long().cpu()
    there = labels >= 0
    picked = torch.log_softmax(x, 1)[there].gather(1, labels[there][:, None])
    loss = -picked.mean()
    loss.backward()
    return float(loss.detach()), [p.grad for p in ps]


def test_gradients_and_parameters_of_a_step():
    el = synth.make_graph("rmat_sparse_stack", scale=0.0003, seed=11)
    widths = (20, 48, 32, 7)
    x = synth.normal_features(el.n, widths[0], 1).to(DEV)
    labels = torch.randint(-3, widths[-1], (el.n,), generator=torch.Generator().manual_seed(2)).clamp(min=-1).to(torch.int32).to(DEV)
    t = train_sage.Trainer(device_graph(el), x, labels, widths, groups=4, embedding=True, lr=1e-2, weight_decay=0.1)
    start = [p.double().cpu() for p in t.params]
    t.step()
    torch.cuda.synchronize()
    loss, grads = reference(el, t, start)
    assert abs(float(t.loss) - loss) <= 1e-5 * abs(loss)
    for g, want in zip(t.grads, grads):
        # sums of some hundred fp32 terms through three layers, and a few gates next to zero that may stand the other way
        off = float((g.double().cpu() - want).norm() / want.norm())
        assert off <= 1e-4, (tuple(g.shape), off)
    # the first step of AdamW: every element by lr g / (|g| + eps), and the decay; where the gradient is not lost in its rounding
    for p, p0, want, decay in zip(t.params, start, grads, [0.0] + [0.1, 0.0, 0.0, 0.0] * 2 + [0.1, 0.0]):
        moved = p0 * (1 - 1e-2 * decay) - 1e-2 * want / (want.abs() + 1e-8)
        sure = want.abs() > 1e-3 * want.abs().max()
        assert float((p.double().cpu() - moved)[sure].abs().max()) <= 2e-4 * 1e-2 + 1e-6 * float(p0.abs().max())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("embedding", [False, True])
def test_training_learns_the_teacher(bits, embedding):
    t = train_sage.make(scale=0.002, widths=(100, 64, 16), labelled=0.5, state_bits=bits, embedding=embedding)
    losses = [float(t.step()) for _ in range(60)]
    assert all(l == l for l in losses) and losses[-1] < 0.6 * losses[0], (losses[0], losses[-1])
    assert all(bool(torch.isfinite(p).all()) for p in t.params)


def test_a_captured_forward_and_backward_pass_repeats_itself():
    t = train_sage.make(scale=0.002, widths=(100, 64, 16), labelled=0.5)
    t.forward()
    t.backward()
    torch.cuda.synchronize()
    want = [t.loss.clone()] + [g.clone() for g in t.grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.forward()
        t.backward()
    for _ in range(3):
        for g in [t.loss] + t.grads:
            g.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [t.loss] + t.grads))
