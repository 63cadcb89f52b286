"""A whole training step in the library's calls, from ids to updated parameters: lookup, norm with a skip connection, loss, their gradients, clipping, AdamW."""
import os
import sys

import pytest
import torch

from paper_2110_08450_amd import binding as smfg

from test_gpu_training_ops import DEV, U, count, gen, ids_of

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu
EPS, LR, MAX_NORM = 1e-5, 1e-2, 0.5


class Model:
    """logits = rms_norm(x + r) W^T of looked-up rows x, all floats; the table's touched rows have states of 8 bits, or of floats."""

    def __init__(self, n, rows, dim, classes, bytes_):
        self.n, self.dim, self.classes = n, dim, classes
        self.table = torch.randn((rows, dim), device=DEV, generator=gen(1))
        self.r = torch.randn((n, dim), device=DEV, generator=gen(2))
        self.w = 1 + 0.1 * torch.randn(dim, device=DEV, generator=gen(3))
        self.out = torch.randn((classes, dim), device=DEV, generator=gen(4)) * dim ** -0.5
        self.ids, self.labels, self.num = ids_of("mixed", n, rows, 5), torch.randint(-1, classes, (n,), device=DEV, generator=gen(6)), count(n)
        self.x, self.t, self.y, self.dx = [torch.zeros((n, dim), device=DEV) for _ in range(4)]
        self.rstd, self.loss, self.norm = torch.zeros(n, device=DEV), torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
        self.dlogits, self.dw, self.dout = torch.zeros((n, classes), device=DEV), torch.empty_like(self.w), torch.empty_like(self.out)
        self.row_ids, self.num_rows, self.rows = torch.zeros(n, dtype=torch.int32, device=DEV), count(0), torch.zeros((n, dim), device=DEV)
        self.ws = [smfg.cross_entropy_workspace(n, classes), smfg.rms_norm_grad_workspace(n, dim), smfg.embedding_grad_workspace(n, rows, dim)]
        self.grads = smfg.grad_list([self.rows, self.dw, self.dout], rows=[self.num_rows, None, None])
        dense = [self.w, self.out]
        if bytes_:
            m, v = torch.zeros((rows, dim), dtype=torch.int8, device=DEV), torch.zeros((rows, dim), dtype=torch.uint8, device=DEV)
            s = [[torch.zeros((rows, -(-dim // smfg.STATE_BLOCK)), device=DEV), None, None] for _ in range(2)]
        else:
            m, v, s = torch.zeros_like(self.table), torch.zeros_like(self.table), [None, None]
        self.m, self.v = [m] + [torch.zeros_like(p) for p in dense], [v] + [torch.zeros_like(p) for p in dense]
        self.step_number = count(0)
        self.params = smfg.adamw_list([self.table] + dense, [self.rows, self.dw, self.dout], self.m, self.v, *s, rows=[self.num_rows, None, None],
                                      row_ids=[self.row_ids, None, None], weight_decay=[0.0, 0.0, 0.1])
        self.states = [self.table, self.w, self.out, self.loss, self.norm, *self.m, *self.v, *[t[0] for t in s if t]]

    def step(self, stream=None):
        n = self.n
        smfg.embedding(self.table, self.ids, self.num, n, self.x, stream=stream)
        smfg.rms_norm(self.x, self.num, n, self.w, EPS, self.y, residual=self.r, total=self.t, rstd=self.rstd, stream=stream)
        torch.mm(self.y, self.out.t(), out=self.dlogits)
        smfg.cross_entropy(self.dlogits, self.labels, self.num, n, self.loss, self.ws[0], grad_logits=self.dlogits, stream=stream)
        torch.mm(self.dlogits.t(), self.y, out=self.dout)
        torch.mm(self.dlogits, self.out, out=self.dx)
        smfg.rms_norm_grad(self.dx, self.t, self.num, n, self.w, self.rstd, self.dx, self.dw, self.ws[1], stream=stream)
        smfg.embedding_grad_rows(self.ids, self.num, n, self.dx, self.table.shape[0], self.row_ids, self.num_rows, self.rows, self.ws[2], stream=stream)
        smfg.clip_grad_norm(self.grads, float("inf"), self.norm, stream=stream)
        self.step_number.add_(1)
        smfg.adamw(self.params, 0, LR, max_norm=MAX_NORM, norm=self.norm, device_step=self.step_number, stream=stream)


def reference(model, steps):
    """Losses and parameters of the same steps in 64 bits, by automatic differentiation; lazy steps of the touched rows."""
    table, w, out = [t.double().clone() for t in (model.table, model.w, model.out)]
    ids, labels, r = model.ids, model.labels, model.r.double()
    inside, live = (ids >= 0) & (ids < table.shape[0]), labels >= 0
    m, v = [[torch.zeros_like(t) for t in (table, w, out)] for _ in range(2)]
    losses, norms = [], []
    for t in range(1, steps + 1):
        p = [x.clone().requires_grad_() for x in (table, w, out)]
        x = torch.where(inside[:, None], p[0][torch.where(inside, ids, 0)], 0.0) + r
        y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * p[1]
        loss = torch.nn.functional.cross_entropy((y @ p[2].t())[live], labels[live])
        grads = torch.autograd.grad(loss, p)
        norm = torch.sqrt(sum((g * g).sum() for g in grads))
        losses.append(loss.item())
        norms.append(norm.item())
        f = min(1.0, MAX_NORM / (norms[-1] + 1e-6))
        touched = torch.zeros(table.shape[0], dtype=torch.bool, device=DEV)
        touched[ids[inside]] = True
        for i, (q, g, decay) in enumerate(zip((table, w, out), grads, (0.0, 0.0, 0.1))):
            rows = touched if i == 0 else slice(None)
            m[i][rows] = 0.9 * m[i][rows] + 0.1 * f * g[rows]
            v[i][rows] = 0.999 * v[i][rows] + 0.001 * (f * g[rows]) ** 2
            q[rows] = q[rows] * (1 - LR * decay) - LR * m[i][rows] / (1 - 0.9 ** t) / (torch.sqrt(v[i][rows] / (1 - 0.999 ** t)) + 1e-8)
    return losses, norms, (table, w, out)


SIZES = [(700, 300, 48, 30), (3000, 2000, 100, 1013)]


@pytest.mark.parametrize("n,rows,dim,classes", SIZES)
def test_steps_follow_64_bits(n, rows, dim, classes):
    """The first step is exact but for roundings of float sums of some thousand terms; where a gradient is near 0 its step of LR m / sqrt(v) turns on its sign, so
    that parameters are compared in the 2-norm: by a rounding of 4096 U of each gradient's size, of LR a step."""
    model = Model(n, rows, dim, classes, False)
    losses, norms, want = reference(model, 3)
    for i in range(3):
        model.step()
        assert abs(float(model.loss) - losses[i]) <= 4096 * U * losses[i] * (1 if i == 0 else 30)
        assert abs(float(model.norm) - norms[i]) <= 4096 * U * norms[i] * (1 if i == 0 else 30)
    for have, q in zip((model.table, model.w, model.out), want):
        assert float((have.double() - q).norm()) <= 0.01 * 3 * LR * q.numel() ** 0.5


@pytest.mark.parametrize("bytes_", [False, True])
def test_a_step_in_a_graph(bytes_):
    """Replays over new inputs, with eager steps of another model between them, give the eager step's bits; the step's number is on the device."""
    n, rows, dim, classes = SIZES[1]
    a, b = Model(n, rows, dim, classes, bytes_), Model(n, rows, dim, classes, bytes_)
    a.step()
    b.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for k in range(4):
        ids = ids_of(("mixed", "uniform", "outside", "same")[k], n, rows, 30 + k)
        labels = torch.randint(-1, classes, (n,), device=DEV, generator=gen(40 + k))
        for s in (a, b):
            s.ids.copy_(ids)
            s.labels.copy_(labels)
            s.num.fill_(n - 500 * k)
        for s in (a, b):  # rows that no longer count keep what the products read
            s.y.zero_()
            s.dlogits.zero_()
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(a.states, b.states)):
            assert torch.equal(x, y), (k, i)
    assert int(a.step_number) == 5


def test_two_graphs_share_their_scratch():
    """Captured with the same scratch, replayed one behind the other and the other way round."""
    n, dim, classes = 2000, 96, 300
    t = torch.randn((n, dim), device=DEV, generator=gen(1))
    x = [torch.randn((n, classes), device=DEV, generator=gen(2 + i)) for i in range(2)]
    y, num = torch.randint(0, classes, (n,), device=DEV, generator=gen(4)), count(n)
    ws, wn = smfg.cross_entropy_workspace(n, classes), smfg.rms_norm_grad_workspace(n, dim)
    rstd = torch.ones(n, device=DEV)
    outs = [[torch.zeros(1, device=DEV), torch.empty_like(x[0]), torch.empty_like(t), torch.empty(dim, device=DEV)] for _ in range(2)]
    eager = [[torch.zeros(1, device=DEV), torch.empty_like(x[0]), torch.empty_like(t), torch.empty(dim, device=DEV)] for _ in range(2)]

    def work(i, o):
        smfg.cross_entropy(x[i], y, num, n, o[0], ws, grad_logits=o[1])
        smfg.rms_norm_grad(t, t, num, n, None, rstd, o[2], o[3], wn)

    graphs = []
    for i in range(2):
        work(i, eager[i])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            work(i, outs[i])
    for order in ((0, 1), (1, 0), (1, 1, 0)):
        for o in outs:
            for a in o:
                a.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(outs[i], eager[i]))


def test_the_example_with_adamw():
    """It runs, its loss is a number, and its states are those of the rows that were touched."""
    import node_embeddings
    model, losses = node_embeddings.train(12, optimizer="adamw", lr=0.01)
    assert all(x == x and x < 10 for x in losses) and model.steps == 12
    m, v, ms, vs = [model.adamw.tensors[i][0] for i in (2, 3, 4, 5)]
    touched = (vs != 0).any(1)
    assert bool(touched.any()) and not bool(v[~touched].any()) and not bool(m[~touched].any()) and bool(ms[touched].isfinite().all())
