"""Gradients that are new tensors in every step."""
import pytest
import torch

import paper_2104_06700_amd as gnn

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(300, 7), (513,), (1,)]


def model(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    params = [torch.randn(s, device=DEV, generator=gen) for s in SIZES]
    return params, [torch.zeros_like(p) for p in params], [torch.zeros_like(p) for p in params]


def gradients(step):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(100 + step)
    return [torch.randn(s, device=DEV, generator=gen) for s in SIZES]


def test_steps_with_new_gradients_equal_those_with_gradients_in_place():
    (p, m, v), (q, n, w) = model(1), model(1)
    kept = [torch.zeros_like(t) for t in p]
    in_place, anew = gnn.AdamWTensors(p, kept, m, v), gnn.AdamWTensors(q, [None] * 3, n, w)
    for step in range(1, 5):
        for t, g in zip(kept, gradients(step)):
            t.copy_(g)
        if step == 3:
            in_place.set_grads([kept[0], None, kept[2]])
        elif step == 4:
            in_place.set_grads(kept)
        gnn.gnn_adamw_step(in_place, step, 1e-2)
        new = gradients(step)
        if step == 3:
            new[1] = None
        anew.set_grads(new)
        del new  # the handle keeps them until the next ones
        gnn.gnn_adamw_step(anew, step, 1e-2)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(p + m + v, q + n + w)), step
    assert not any(torch.equal(a, b) for a, b in zip(p, model(1)[0]))


def test_wrong_gradients_are_refused_and_the_ones_before_stay():
    p, m, v = model(2)
    g = gradients(1)
    tensors = gnn.AdamWTensors(p, g, m, v)
    for bad, error in (([g[0], g[1]], ValueError), ([g[0], g[1], g[1]], ValueError), ([g[0].bfloat16(), g[1], g[2]], TypeError),
                       ([g[0].cpu(), g[1], g[2]], ValueError), ([g[0].t(), g[1], g[2]], ValueError)):
        with pytest.raises(error):
            tensors.set_grads(bad)
    before = [t.clone() for t in p]
    gnn.gnn_adamw_step(tensors, 1, 1e-2)
    torch.cuda.synchronize()
    # the first step: every element by the rate, against its gradient
    for a, b, t in zip(p, before, g):
        assert float((a - (b - 1e-2 * t.sign())).abs().max()) < 1e-5
