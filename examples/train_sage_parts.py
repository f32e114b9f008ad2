"""Training of a GraphSAGE model a part of the vertices at a time: each step takes the vertices of one part and the neighbours that they have
outside it.

    python examples/train_sage_parts.py                               # 24 thousand vertices in 8 parts
    python examples/train_sage_parts.py --scale 1.0 --parts 16        # 2.4 million vertices
    python examples/train_sage_parts.py --embedding --muon            # learned vertex embeddings; weight matrices by Muon

A step looks the input rows of its vertices up in the table of all.  Hidden rows of neighbours outside the part are not computed: every step
keeps the hidden rows of its own vertices, in 8 bits, and reads those of the others as the last step of their part left them.  With
learned embeddings the gradients of the rows that were looked up are summed into that of the table.  Every part's graph is built once, and
everything that a step needs is allocated once.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
for _p in (HERE, os.path.dirname(HERE)):
    if _p not in sys.path:
        sys.path.insert(0, _p)

import paper_2104_06700_amd as gnn  # noqa: E402
import train_sage  # noqa: E402


class Part:
    """Vertices lo .. hi - 1, then those outside that they have edges from: the edges into the former, with the numbers of this list."""

    def __init__(self, dst, src, lo, hi, labels):
        there = (dst >= lo) & (dst < hi)
        d, s = dst[there].long() - lo, src[there].long()
        own = (s >= lo) & (s < hi)
        outside = torch.unique(s[~own])
        s = torch.where(own, s - lo, torch.searchsorted(outside, s) + (hi - lo))
        self.own, self.n = hi - lo, hi - lo + outside.numel()
        order = torch.argsort(d * self.n + s)
        self.graph = gnn.build_device_graph(d[order].to(torch.int32), s[order].to(torch.int32), self.n)
        self.ids = torch.cat([torch.arange(lo, hi, device=dst.device), outside]).to(torch.int32)
        self.labels = torch.full((self.n,), -1, device=dst.device, dtype=torch.int32)
        self.labels[:self.own] = labels[lo:hi]


class PartTrainer(train_sage.Trainer):
    """A model whose steps are of one part each."""

    def __init__(self, parts, x, labels, widths, embedding=False, **kw):
        """x [N, F] is a row a vertex: a parameter with `embedding`, else the input features."""
        self.parts, self.table = parts, x
        most = max(parts, key=lambda p: p.n)
        # layers and their room for the part with the most vertices; the other parts have the first rows
        super().__init__(most.graph, torch.empty(most.n, x.shape[1], device=x.device), labels, widths, embedding=embedding, **kw)
        for p in parts:
            for fi, fo in zip(widths, widths[1:]):
                p.graph.plan_fwd.prepare(p.graph.indices, gnn.GNN_SAGE_GCN, False, min(fi, fo))
                p.graph.plan_bwd.prepare(p.graph.indices_t, gnn.GNN_SAGE_GCN, True, min(fi, fo))
        for l in self.layers[:-1]:  # (all zeros reads as rows of zeros)
            l["store"] = torch.zeros(x.shape[0], gnn.gnn_store_row_bytes(l["w"].shape[1]), device=x.device, dtype=torch.uint8)
        room = max(gnn.gnn_lookup_workspace_bytes(x.shape[0], p.n, x.shape[1]) for p in parts)
        for p in parts:
            for fi, fo in zip(widths, widths[1:]):
                room = max(room, gnn.gnn_sage_layer_workspace_bytes(p.n, fi, fo, False), gnn.gnn_softmax_xent_workspace_bytes(p.n, widths[-1]))
                if fo != widths[-1]:
                    room = max(room, gnn.gnn_group_norm_workspace_bytes(p.own, fo, self.groups, 1, True))
        if room > self.workspace.numel():
            self.workspace = torch.empty(room, device=x.device, dtype=torch.uint8)

    def optimizer(self, embedding, bits, weight_decay, muon):
        x, dx = self.x, self.dx
        if embedding:  # the parameter is the table, not the rows of a step
            self.x, self.dx = self.table, torch.empty_like(self.table)
        super().optimizer(embedding, bits, weight_decay, muon)
        self.dtable, self.x, self.dx = self.dx, x, dx

    def forward(self, p):
        x = self.x[:p.n]
        gnn.gnn_lookup_fwd(self.table, p.ids, x)
        for l in self.layers:
            h = l["h"][:p.n]
            gnn.gnn_sage_layer_fwd(p.graph.indptr, p.graph.indices, x, l["w"], l["b"], l["saved"], h, p.graph.plan_fwd, relu=False)
            x = h
            if not l["last"]:
                x = l["y"][:p.n]
                gnn.gnn_group_norm_fwd(h[:p.own], l["gamma"], l["beta"], x[:p.own], l["mean"], l["rstd"], self.groups, act=gnn.GNN_ACT_RELU,
                                       workspace=self.workspace)
                if p.n > p.own:
                    gnn.gnn_load_rows(l["store"], x[p.own:], p.ids[p.own:])
                gnn.gnn_store_rows(x[:p.own], l["store"], p.ids[:p.own], unique=True)
        gnn.gnn_softmax_xent(x, p.labels, self.loss, self.layers[-1]["dh"][:p.n], workspace=self.workspace)

    def backward(self, p):
        for i in reversed(range(len(self.layers))):
            l = self.layers[i]
            h, dh = l["h"][:p.n], l["dh"][:p.n]
            if not l["last"]:  # the rows from outside are constants
                gnn.gnn_group_norm_bwd(h[:p.own], l["gamma"], l["beta"], l["mean"], l["rstd"], l["dy"][:p.own], dh[:p.own], l["dgamma"], l["dbeta"],
                                       self.groups, act=gnn.GNN_ACT_RELU, workspace=self.workspace)
                dh[p.own:].zero_()
            x, dx = (self.layers[i - 1]["y"], self.layers[i - 1]["dy"]) if i else (self.x, self.dx)
            gnn.gnn_sage_layer_bwd(p.graph.indptr_t, p.graph.indices_t, x[:p.n], l["w"], l["saved"], h, dh, None if dx is None else dx[:p.n], l["dw"],
                                   l["db"], p.graph.plan_bwd, self.workspace, relu=False)
        if self.dx is not None:
            gnn.gnn_lookup_bwd(p.ids, self.dx[:p.n], self.dtable, workspace=self.workspace)

    def step(self, p):
        """One step with the vertices of p; the loss is that of the parameters before it, on the device."""
        self.forward(p)
        self.backward(p)
        self.steps += 1
        self.update()
        return self.loss


def cut(dst, src, n, labels, count):
    """Parts of equal numbers of neighbouring vertices."""
    ends = [n * k // count for k in range(count + 1)]
    return [Part(dst, src, lo, hi, labels) for lo, hi in zip(ends, ends[1:])]


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--scale", type=float, default=0.01, help="of the 2,449,029 vertices and 123.7 million edges")
    ap.add_argument("--widths", default="100,256,256,47")
    ap.add_argument("--groups", type=int, default=8)
    ap.add_argument("--parts", type=int, default=8)
    ap.add_argument("--epochs", type=int, default=5)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--embedding", action="store_true", help="the input features are parameters")
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    ap.add_argument("--muon", action="store_true", help="weight matrices by Muon, the rest by AdamW")
    ap.add_argument("--muon-lr", type=float, default=2e-2)
    a = ap.parse_args()
    widths = tuple(int(f) for f in a.widths.split(","))
    dst, src, x, labels = train_sage.data(a.scale, widths)[1:]
    parts = cut(dst, src, x.shape[0], labels, a.parts)
    t = PartTrainer(parts, x, labels, widths, groups=a.groups, lr=a.lr, embedding=a.embedding, state_bits=a.state_bits, muon=a.muon, muon_lr=a.muon_lr)
    print(f"{x.shape[0]} vertices, {src.numel()} edges, parts with up to {max(p.n for p in parts)} vertices", flush=True)
    for k in range(a.epochs):
        torch.cuda.synchronize()
        began = time.perf_counter()
        losses = [t.step(p).clone() for p in parts]
        torch.cuda.synchronize()
        print(f"epoch {k + 1}: loss {float(torch.stack(losses).mean()):.4f}  {1e3 * (time.perf_counter() - began):.2f} ms", flush=True)


if __name__ == "__main__":
    main()
