"""Learned node embeddings under one GraphSAGE layer, trained on sampled batches: the operators of a training step together.

The nodes have no features; a table of floats, a row per node, is learned instead.  One step:

  sample_mfg           the batch: seeds, their sampled neighbours, one block
  embedding            x = scale * table[node ids]
  layer_norm           z = norm(x)
  mean_aggregate       m = mean of z over each seed's neighbours
                       logits = relu([z of the seeds | m] W1 + b1) W2 + b2, cross entropy        (torch)
  embedding_grad       gradient of z: that of the seeds' own rows, and to it the share of every edge's source (accumulate)
  layer_norm_grad      gradients of x, weight and bias
  embedding_grad_rows  the touched rows of the table's gradient
  clip_grad_norm       all gradients together, the touched rows among them
                       plain gradient descent

No size that depends on the batch leaves the GPU, so a step does not wait for it.

    python examples/node_embeddings.py --steps 200
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_2110_08450_amd import binding as smfg  # noqa: E402
from paper_2110_08450_amd import synth  # noqa: E402


class NodeEmbeddings:
    def __init__(self, g: smfg.Graph, batch_size: int, fanout: int, dim: int, hidden: int, classes: int, lr: float = 0.5,
                 max_norm: float = 1.0, seed: int = 0):
        dev = g.indptr.device
        gen = torch.Generator(device=dev).manual_seed(seed)

        def rand(*shape, spread):
            return torch.randn(shape, device=dev, generator=gen) * spread

        self.g, self.fanouts, self.dim, self.lr, self.max_norm = g, (fanout,), dim, lr, max_norm
        self.scale = dim ** 0.5  # rows of the table have unit length or so, what the norm sees unit spread
        self.table = rand(g.num_nodes, dim, spread=dim ** -0.5)
        self.weight, self.bias = torch.ones(dim, device=dev), torch.zeros(dim, device=dev)
        self.w1, self.b1 = rand(2 * dim, hidden, spread=(2 * dim) ** -0.5), torch.zeros(hidden, device=dev)
        self.w2, self.b2 = rand(hidden, classes, spread=hidden ** -0.5), torch.zeros(classes, device=dev)
        # buffers for the largest batch, kept from step to step
        self.ws = smfg.workspace_create(g, batch_size, self.fanouts)
        self.out = smfg.alloc_output(g, batch_size, self.fanouts, with_features=False)
        n, e = self.out.node_capacity, self.out.edge_capacity[0]
        self.n, self.e, self.batch = n, e, batch_size
        self.x, self.z, self.dz = [torch.zeros((n, dim), device=dev) for _ in range(3)]
        self.mean, self.rstd = torch.empty(n, device=dev), torch.empty(n, device=dev)
        self.m = torch.empty((batch_size, dim), device=dev)
        self.row_ids = torch.zeros(n, dtype=torch.int32, device=dev)
        self.num_rows = torch.zeros(1, dtype=torch.int64, device=dev)
        self.rows = torch.zeros((n, dim), device=dev)
        self.grads = [torch.empty_like(p) for p in self.dense()]
        self.norm = torch.zeros(1, device=dev)
        self.ws_norm = smfg.layer_norm_grad_workspace(n, dim)
        self.ws_edges = smfg.embedding_grad_workspace(e, n, dim)
        self.ws_rows = smfg.embedding_grad_workspace(n, g.num_nodes, dim)
        self.all_grads = smfg.grad_list([self.rows] + self.grads, rows=[self.num_rows] + [None] * len(self.grads))

    def dense(self):
        return [self.weight, self.bias, self.w1, self.b1, self.w2, self.b2]

    def gradients(self, seeds: torch.Tensor, labels: torch.Tensor, rng_key: int) -> torch.Tensor:
        """One batch forward and back: the loss; gradients in self.rows (of self.row_ids, self.num_rows of them) and self.grads."""
        s, d = seeds.numel(), self.dim
        smfg.sample_mfg(self.g, self.ws, seeds, self.fanouts, rng_key, self.out)
        nodes, edges = self.out.counts[1:2], self.out.counts[2:3]
        ids, indptr, indices = self.out.node_ids, self.out.indptr[0], self.out.indices[0]

        smfg.embedding(self.table, ids, nodes, self.n, self.x, scale=self.scale)
        smfg.layer_norm(self.x, nodes, self.n, self.weight, self.bias, 1e-5, self.z, self.mean, self.rstd)
        smfg.mean_aggregate(indptr, indices, self.out.counts[0:1], s, self.z, self.m)
        h = torch.cat([self.z[:s], self.m[:s]], 1)
        a = torch.relu(h @ self.w1 + self.b1)
        logp = torch.log_softmax(a @ self.w2 + self.b2, 1)
        loss = -logp.gather(1, labels[:, None]).mean()

        dlogits = logp.exp()
        dlogits[torch.arange(s, device=seeds.device), labels] -= 1
        dlogits /= s
        da = (dlogits @ self.w2.t()) * (a > 0)
        dh = da @ self.w1.t()
        gw, gb, gw1, gb1, gw2, gb2 = self.grads
        torch.mm(h.t(), da, out=gw1)
        torch.sum(da, 0, out=gb1)
        torch.mm(a.t(), dlogits, out=gw2)
        torch.sum(dlogits, 0, out=gb2)
        # the mean's gradient: every edge brings its seed's row, divided by the seed's number of edges, to its source
        start = indptr[:s + 1].long()
        at = torch.searchsorted(start[1:], torch.arange(self.e, device=seeds.device), right=True).clamp_(max=s - 1)
        share = (dh[:, d:] / (start[1:] - start[:-1]).clamp(min=1)[:, None])[at]
        self.dz.zero_()
        self.dz[:s] = dh[:, :d]
        smfg.embedding_grad(indices, edges, self.e, share, self.dz, self.ws_edges, accumulate=True)
        smfg.layer_norm_grad(self.dz, self.x, nodes, self.n, self.weight, self.mean, self.rstd, self.dz, gw, gb, self.ws_norm)
        smfg.embedding_grad_rows(ids, nodes, self.n, self.dz, self.g.num_nodes, self.row_ids, self.num_rows, self.rows, self.ws_rows, scale=self.scale)
        return loss

    def step(self, seeds: torch.Tensor, labels: torch.Tensor, rng_key: int) -> torch.Tensor:
        loss = self.gradients(seeds, labels, rng_key)
        smfg.clip_grad_norm(self.all_grads, self.max_norm, self.norm)
        for p, g in zip(self.dense(), self.grads):
            p.sub_(g, alpha=self.lr)
        used = torch.arange(self.n, device=seeds.device) < self.num_rows  # rows behind them hold what an earlier batch left
        self.table.index_add_(0, torch.where(used, self.row_ids, 0), torch.where(used[:, None], self.rows, 0.0), alpha=-self.lr)
        return loss


def train(steps: int, dim: int = 64, hidden: int = 128, classes: int = 16, fanout: int = 10, report=None):
    """Trains on the seed batches of the smallest workload with random labels, which only a row per node can learn; the losses."""
    dev = "cuda:0"
    w = synth.WORKLOADS["tiny"]
    graph = synth.make_graph(w, device=dev)
    g = smfg.graph_create(graph.indptr, graph.indices)
    batches = synth.make_seed_batches(w, device=dev)
    labels = torch.randint(0, classes, (w.num_nodes,), device=dev, generator=torch.Generator(device=dev).manual_seed(1))
    model = NodeEmbeddings(g, w.batch_size, fanout, dim, hidden, classes)
    losses = []
    for i in range(steps):
        seeds = batches[i % len(batches)]
        losses.append(model.step(seeds, labels[seeds.long()], synth.batch_rng_key(w, i)))
        if report and (i + 1) % 20 == 0:
            report(f"step {i + 1}: loss {float(losses[-1]):.4f}, gradient norm {float(model.norm):.3f}, {int(model.num_rows)} rows touched")
    return model, [float(x) for x in losses]


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=200)
    p.add_argument("--dim", type=int, default=64)
    a = p.parse_args()
    losses = train(a.steps, dim=a.dim, report=lambda s: print(s, flush=True))[1]
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
