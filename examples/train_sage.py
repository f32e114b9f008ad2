"""Full-batch training of a GraphSAGE model with the library's calls only: layers, group norm with a rectifier between them, the loss
of the labelled vertices and AdamW over all parameters.

    python examples/train_sage.py                                   # 24 thousand vertices, three layers
    python examples/train_sage.py --scale 1.0 --steps 5             # 2.4 million vertices
    python examples/train_sage.py --embedding --state-bits 8        # learned vertex embeddings, optimizer states in 8 bits
    python examples/train_sage.py --muon                            # weight matrices by orthogonalised updates, the rest by AdamW

The graph is a seeded synthetic one; the labels are those of a random teacher on the aggregated features, so there is something to
learn.  Everything a step needs is allocated once; a step is nothing but library calls.
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2104_06700_amd as gnn  # noqa: E402
import synth  # noqa: E402


class Trainer:
    """Parameters, activations, gradients and states of a model on one graph."""

    def __init__(self, graph, x, labels, widths, groups=8, embedding=False, state_bits=32, lr=1e-2, weight_decay=1e-2, seed=0, muon=False,
                 muon_lr=2e-2):
        self.g, self.x, self.labels, self.widths, self.groups, self.lr, self.muon_lr = graph, x, labels, widths, groups, lr, muon_lr
        n, dev = graph.n, x.device
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed)

        def new(*shape):
            return torch.empty(shape, device=dev)
        self.layers, room = [], 0
        for i, (fi, fo) in enumerate(zip(widths, widths[1:])):
            last = i + 2 == len(widths)
            l = dict(w=new(fi, fo).normal_(generator=gen) / math.sqrt(fi), b=torch.zeros(fo, device=dev), dw=new(fi, fo), db=new(fo),
                     saved=new(gnn.gnn_sage_layer_saved_elems(n, fi, fo)), h=new(n, fo), dh=new(n, fo), last=last)
            if not last:  # group norm and rectifier behind every layer but the last
                l.update(gamma=torch.ones(fo, device=dev), beta=torch.zeros(fo, device=dev), dgamma=new(fo), dbeta=new(fo), mean=new(1, groups),
                         rstd=new(1, groups), y=new(n, fo), dy=new(n, fo))
                room = max(room, gnn.gnn_group_norm_workspace_bytes(n, fo, groups, 1, True))
            room = max(room, gnn.gnn_sage_layer_workspace_bytes(n, fi, fo, False))
            f = min(fi, fo)
            graph.plan_fwd.prepare(graph.indices, gnn.GNN_SAGE_GCN, False, f)
            graph.plan_bwd.prepare(graph.indices_t, gnn.GNN_SAGE_GCN, True, f)
            self.layers.append(l)
        self.dx = torch.empty_like(x) if embedding else None
        room = max(room, gnn.gnn_softmax_xent_workspace_bytes(n, widths[-1]))
        self.loss = new(1)
        self.optimizer(embedding, state_bits, weight_decay, muon)
        if self.muon is not None:
            room = max(room, gnn.gnn_muon_workspace_bytes(self.muon))
        self.workspace = torch.empty(room, device=dev, dtype=torch.uint8)

    def optimizer(self, embedding, bits, weight_decay, muon):
        """Weights (decayed) and embeddings hold AdamW's states in `bits` bits, vectors in 32; with muon the weights have a momentum instead."""
        params, grads, decay = [], [], []
        if embedding:
            params, grads, decay = [self.x], [self.dx], [0.0]
        for l in self.layers:
            params += [l["w"], l["b"]]
            grads += [l["dw"], l["db"]]
            decay += [weight_decay, 0.0]
            if not l["last"]:
                params += [l["gamma"], l["beta"]]
                grads += [l["dgamma"], l["dbeta"]]
                decay += [0.0, 0.0]
        self.params, self.grads, self.muon = params, grads, None
        if muon:
            self.momentum = [torch.zeros_like(l["w"]) for l in self.layers]
            self.muon = gnn.MuonTensors([l["w"] for l in self.layers], [l["dw"] for l in self.layers], self.momentum, weight_decay=weight_decay)
            weights = [id(l["w"]) for l in self.layers]
            params, grads, decay = zip(*[t for t in zip(params, grads, decay) if id(t[0]) not in weights])
        m, v, ms, vs = [], [], [], []
        for p in params:
            eight = bits == 8 and p.dim() == 2
            for states, scales in ((m, ms), (v, vs)):
                states.append(torch.zeros(p.shape, device=p.device).to(torch.float8_e4m3fn) if eight else torch.zeros_like(p))
                scales.append(torch.zeros(-(-p.numel() // gnn.GNN_ADAMW_BLOCK), device=p.device) if eight else None)
        self.tensors = gnn.AdamWTensors(params, grads, m, v, ms, vs, weight_decay=decay)
        self.steps = 0

    def forward(self):
        x = self.x
        for l in self.layers:
            gnn.gnn_sage_layer_fwd(self.g.indptr, self.g.indices, x, l["w"], l["b"], l["saved"], l["h"], self.g.plan_fwd, relu=False)
            x = l["h"]
            if not l["last"]:
                gnn.gnn_group_norm_fwd(l["h"], l["gamma"], l["beta"], l["y"], l["mean"], l["rstd"], self.groups, act=gnn.GNN_ACT_RELU, workspace=self.workspace)
                x = l["y"]
        gnn.gnn_softmax_xent(x, self.labels, self.loss, self.layers[-1]["dh"], workspace=self.workspace)

    def backward(self):
        for i in reversed(range(len(self.layers))):
            l = self.layers[i]
            if not l["last"]:
                gnn.gnn_group_norm_bwd(l["h"], l["gamma"], l["beta"], l["mean"], l["rstd"], l["dy"], l["dh"], l["dgamma"], l["dbeta"], self.groups,
                                       act=gnn.GNN_ACT_RELU, workspace=self.workspace)
            x, dx = (self.layers[i - 1]["y"], self.layers[i - 1]["dy"]) if i else (self.x, self.dx)
            gnn.gnn_sage_layer_bwd(self.g.indptr_t, self.g.indices_t, x, l["w"], l["saved"], l["h"], l["dh"], dx, l["dw"], l["db"], self.g.plan_bwd,
                                   self.workspace, relu=False)

    def step(self):
        """One step; the loss is that of the parameters before it, on the device."""
        self.forward()
        self.backward()
        self.steps += 1
        self.update()
        return self.loss

    def update(self):
        gnn.gnn_adamw_step(self.tensors, self.steps, self.lr)
        if self.muon is not None:
            gnn.gnn_muon_step(self.muon, self.muon_lr, workspace=self.workspace)


def data(scale, widths, labelled=0.08, seed=3, device="cuda:0"):
    """The synthetic 2.4-million-vertex graph times `scale`, its edges, features and labels."""
    el = synth.make_graph("rmat_sparse_stack", device=device, scale=scale, seed=seed)
    graph = gnn.build_device_graph(el.dst, el.src, el.n)
    x = synth.normal_features(el.n, widths[0], seed, device=device)
    # the teacher: the class of the largest of random projections of the aggregated features
    z, scores = torch.empty_like(x), torch.empty(el.n, widths[-1], device=device)
    gnn.gnn_aggregate_fwd(graph.indptr, graph.indices, None, x, z, el.n, widths[0], gnn.GNN_SAGE_GCN, plan=graph.plan_fwd)
    gnn.gnn_matmul(z, synth.normal_features(widths[0], widths[-1], seed + 1, device=device), scores)
    labels = scores.argmax(1).to(torch.int32)
    labels[synth.uniform_features(el.n, 1, seed + 2, device=device).view(-1) >= 2 * labelled - 1] = -1
    return graph, el.dst, el.src, x, labels


def make(scale=0.01, widths=(100, 256, 256, 47), labelled=0.08, seed=3, device="cuda:0", **kw):
    """A trainer on the synthetic graph."""
    graph, _, _, x, labels = data(scale, widths, labelled, seed, device)
    return Trainer(graph, x, labels, widths, **kw)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--scale", type=float, default=0.01, help="of the 2,449,029 vertices and 123.7 million edges")
    ap.add_argument("--widths", default="100,256,256,47")
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--embedding", action="store_true", help="the input features are parameters too")
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--muon", action="store_true", help="weight matrices by Muon, the rest by AdamW")
    ap.add_argument("--muon-lr", type=float, default=2e-2)
    a = ap.parse_args()
    t = make(a.scale, tuple(int(f) for f in a.widths.split(",")), groups=a.groups, lr=a.lr, embedding=a.embedding, state_bits=a.state_bits,
             muon=a.muon, muon_lr=a.muon_lr)
    print(f"{t.g.n} vertices, {t.g.e} edges, {sum(p.numel() for p in t.params)} parameters", flush=True)
    for k in range(a.steps):
        torch.cuda.synchronize()
        began = time.perf_counter()
        loss = t.step()
        torch.cuda.synchronize()
        print(f"step {k + 1}: loss {float(loss):.4f}  {1e3 * (time.perf_counter() - began):.2f} ms", flush=True)


if __name__ == "__main__":
    main()
