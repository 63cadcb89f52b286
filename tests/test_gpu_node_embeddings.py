"""The training example: its gradients against automatic differentiation in 64 bits, and that it learns."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))
import node_embeddings  # noqa: E402

from paper_2110_08450_amd import binding as smfg  # noqa: E402
from paper_2110_08450_amd import synth  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradients_of_a_batch():
    """Float sums of at most some thousand terms: within 2^-24 times that of the gradients' sizes, in the 2-norm."""
    w = synth.WORKLOADS["tiny"]
    graph = synth.make_graph(w, device=DEV)
    g = smfg.graph_create(graph.indptr, graph.indices)
    seeds = synth.make_seed_batches(w, device=DEV)[0]
    labels = torch.randint(0, 7, (seeds.numel(),), device=DEV, generator=torch.Generator(device=DEV).manual_seed(2))
    model = node_embeddings.NodeEmbeddings(g, w.batch_size, 5, 36, 24, 7)
    loss = model.gradients(seeds, labels, 77)
    n0, n1, e, status = smfg.read_counts(model.out)
    assert status == 0 and n0 == seeds.numel()
    ids, indptr, indices = [t.cpu().long() for t in (model.out.node_ids[:n1], model.out.indptr[0][:n0 + 1], model.out.indices[0][:e])]
    p = [t.cpu().double().requires_grad_() for t in [model.table] + model.dense()]
    table, weight, bias, w1, b1, w2, b2 = p
    x = model.scale * table[ids]
    c = x - x.mean(1, keepdim=True)
    z = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * weight + bias
    k = indptr[1:] - indptr[:-1]
    at = torch.repeat_interleave(torch.arange(n0), k)
    m = torch.zeros((n0, 36), dtype=torch.float64).index_add(0, at, z[indices]) / k.clamp(min=1)[:, None]
    a = torch.relu(torch.cat([z[:n0], m], 1) @ w1 + b1)
    want = torch.nn.functional.cross_entropy(a @ w2 + b2, labels.cpu())
    want.backward()
    assert abs(float(loss) - want.item()) <= 4096 * 2.0 ** -24 * want.item()
    u = int(model.num_rows)
    rows = model.row_ids[:u].cpu().long()
    assert torch.equal(rows, torch.unique(ids))
    got = torch.zeros_like(table.grad)
    got[rows] = model.rows[:u].cpu().double()
    for have, t in zip([got] + [q.cpu().double() for q in model.grads], p):
        assert torch.linalg.vector_norm(have - t.grad) <= 4096 * 2.0 ** -24 * torch.linalg.vector_norm(t.grad)


def test_training_learns():
    """Random labels of the seeds are learned by their rows; gradients are clipped on the way."""
    model, losses = node_embeddings.train(120)
    assert losses[0] > 2.5 and losses[-1] < 0.5 * losses[0] and all(x == x for x in losses)
