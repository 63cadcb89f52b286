"""Performance cases of the training operators on one MI355X: embedding lookup and its gradient, layer norm and its
gradient, the clipping of gradients by their global norm.

A case is a dict of plain values.  Five kinds of work, each through the package's public calls:

  embed       embedding: scaled rows of a table by id
  embed_grad  embedding_grad (form "dense": the whole table's gradient, "add": added to one) or embedding_grad_rows
              (form "rows": the touched rows alone)
  norm        layer_norm with the statistics that its gradient needs
  norm_grad   layer_norm_grad: gradients of the input, the weight and the bias
  clip        clip_grad_norm: global norm, and the gradients scaled into the buffers that an optimizer reads

As everywhere in the package, the number of rows in use lives on the device, and buffers have room for more.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
SIZE = {"f16": 2, "bf16": 2, "f32": 4, "i32": 4, "i64": 8}
EPS = 1e-5


def listed():
    return [
        # learned features for the 16 nodes of a prediction request on a products-sized graph: latency
        dict(name="embed_request", kind="embed", rows=2_450_000, dim=100, table="f16", out="f16", ids=16, cap=16, id="i32", law="uniform",
             scale=1.0),
        # learned features of the final frontier of a batch: float table, half rows for the layers; an eighth of the papers100M shape
        dict(name="embed_frontier", kind="embed", rows=13_900_000, dim=128, table="f32", out="f16", ids=540_000, cap=600_000, id="i32",
             law="uniform", scale=1.0),
        # gradient of a toy data set's small batch, added to what earlier micro-batches left: latency
        dict(name="grad_tiny", kind="embed_grad", form="add", rows=10_000, dim=32, dy="f32", grad="f32", ids=256, cap=256, id="i32",
             law="uniform", scale=1.0),
        # gradient of a token embedding, a few ids very frequent, rows scaled by sqrt(dim): the whole table is written
        dict(name="grad_tokens", kind="embed_grad", form="dense", rows=50_000, dim=1024, dy="bf16", grad="f32", ids=16_384, cap=16_384, id="i64",
             law="zipf", scale=32.0),
        # gradient of node embeddings through the edges of a products-sized block: touched rows alone
        dict(name="grad_edges", kind="embed_grad", form="rows", rows=2_450_000, dim=100, dy="f16", grad="f32", ids=480_000, cap=500_000, id="i32",
             law="zipf", scale=1.0),
        # gradient of label embeddings (a row per class): few rows, each the sum of a thousand
        dict(name="grad_labels", kind="embed_grad", form="dense", rows=172, dim=256, dy="f16", grad="f32", ids=154_321, cap=180_224, id="i32",
             law="uniform", scale=1.0),
        # the norm before the last layer, one row per seed: latency
        dict(name="norm_seeds", kind="norm", rows=1024, cap=1024, dim=256, x="f16", par="f32", spare=0),
        # the norm between the first layers, a row per node of the middle frontier
        dict(name="norm_hidden", kind="norm", rows=154_321, cap=180_224, dim=256, x="f16", par="f32", spare=0),
        # gradient over the raw features' odd width, rows in a wider buffer
        dict(name="norm_grad_odd", kind="norm_grad", rows=47_062, cap=50_000, dim=301, x="f32", par="f32", spare=19),
        # gradient of wide hidden states, parameters of the same type
        dict(name="norm_grad_wide", kind="norm_grad", rows=16_384, cap=16_384, dim=4096, x="bf16", par="bf16", spare=0),
        # all gradients of a three-layer GraphSAGE, clipped into an optimizer's buffers: latency
        dict(name="clip_sage", kind="clip", tensors=9, total=280_748, g="f32", out="f32", scale=1.0, max_norm=1.0),
        # all half gradients of a large model, unscaled and clipped into float ones
        dict(name="clip_large", kind="clip", tensors=290, total=400_000_000, g="f16", out="f32", scale=1.0 / 1024, max_norm=1.0),
    ]


# ---- cases drawn from the same ranges ------------------------------------------------------------

def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _dim(rng):
    return rng.choice([rng.randint(1, 700), 8 * rng.randint(1, 64), rng.choice([32, 100, 128, 172, 256]), 1024 * rng.choice([1, 2, 4, 5, 6, 8])])


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "norm", "norm_grad", "clip"])
    while True:
        if kind == "clip":
            g = rng.choice(["f16", "bf16", "f32"])
            c = dict(kind=kind, tensors=_log(rng, 1, 400), total=_log(rng, 10_000, 390_000_000), g=g, out=rng.choice([g, "f32"]),
                     scale=rng.choice([1.0, 1.0 / 8, 1.0 / 1024]), max_norm=rng.choice([0.5, 1.0, 1e9]))
            if c["total"] >= 4 * c["tensors"]:
                return c
        elif kind in ("norm", "norm_grad"):
            x = rng.choice(["f16", "bf16", "f32"])
            dim = _dim(rng)
            n = _log(rng, 1, max(4, min(200_000, 130_000_000 // dim)))
            return dict(kind=kind, rows=n, cap=n + rng.choice([0, 0, rng.randint(1, 1 + n // 4)]), dim=dim, x=x, par=rng.choice([x, "f32"]),
                        spare=rng.choice([0, 0, rng.randint(1, 64)]))
        else:
            dim = _dim(rng)
            t = rng.choice(["f16", "bf16", "f32"])
            rows = _log(rng, 4, 14_000_000)
            n = _log(rng, 1, max(4, min(900_000, 130_000_000 // dim)))
            c = dict(kind=kind, rows=rows, dim=dim, ids=n, cap=n + rng.choice([0, rng.randint(1, 1 + n // 4)]), id=rng.choice(["i32", "i64"]),
                     law=rng.choice(["uniform", "zipf"]), scale=rng.choice([1.0, math.sqrt(dim)]))
            if kind == "embed":
                c.update(table=t, out=rng.choice([t] + ["f16", "bf16"] * (t == "f32")))
                if rows * dim * SIZE[t] < 7_200_000_000:
                    return c
            else:
                c.update(dy=t, grad=rng.choice(["f32", t]), form=rng.choice(["dense", "add", "rows"]))
                if c["form"] == "add":
                    c["grad"] = "f32"  # many passes are added up
                if (rows if c["form"] != "rows" else c["cap"]) * dim * SIZE[c["grad"]] < 2_400_000_000:
                    return c


# ---- inputs --------------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 16 + salt)


def _randn(shape, dtype, gen, mul=1.0):
    return torch.randn(shape, device=DEV, dtype=torch.float32, generator=gen).mul_(mul).to(DTYPES[dtype])


def _ids(c, seed):
    """Ids of a table: evenly spread, or the rank r with probability about 1 / r, ranks spread over the table.  Four in a thousand are
    -1: a padded place."""
    gen = _gen(seed, 1)
    u = torch.rand(c["cap"], device=DEV, dtype=torch.float64, generator=gen)
    n = c["rows"]
    if c["law"] == "zipf":
        r = torch.exp(u * math.log(n + 1)).to(torch.int64).sub_(1).clamp_(0, n - 1)
        r = (r * 2_654_435_761 + 12_345) % n
    else:
        r = (u * n).to(torch.int64).clamp_(0, n - 1)
    r[torch.rand(c["cap"], device=DEV, generator=gen) < 0.004] = -1
    return r.to(DTYPES[c["id"]])


def _count(n):
    return torch.tensor([n], dtype=torch.int64, device=DEV)


def _sizes(c):
    """Lengths of the tensors of a model: matrices of a few sizes, each with a vector or two behind it, the last takes the rest."""
    n, total = c["tensors"], c["total"]
    w = [(1.0, 0.003, 0.25, 0.002, 0.7)[i % 5] for i in range(n)]
    s = [max(1, int(total * x / sum(w)) - (i % 3)) for i, x in enumerate(w)]
    s[0] += total - sum(s)
    return s


def _views(flat, sizes):
    return [v for v in torch.split(flat, sizes)]


def prepare(case, seed):
    c, k = case, case["kind"]
    s = {"case": c}
    if k == "embed":
        s.update(table=_randn((c["rows"], c["dim"]), c["table"], _gen(seed, 2)), ids=_ids(c, seed), n=_count(c["ids"]),
                 out=torch.zeros((c["cap"], c["dim"]), dtype=DTYPES[c["out"]], device=DEV))
    elif k == "embed_grad":
        s.update(ids=_ids(c, seed), n=_count(c["ids"]), dy=_randn((c["cap"], c["dim"]), c["dy"], _gen(seed, 2), 0.01))
        if c["form"] == "rows":
            s.update(row_ids=torch.full((c["cap"],), -1, dtype=torch.int32, device=DEV), num=_count(0),
                     grad=torch.zeros((c["cap"], c["dim"]), dtype=DTYPES[c["grad"]], device=DEV))
        else:
            s.update(grad=_randn((c["rows"], c["dim"]), c["grad"], _gen(seed, 3), 0.01))
    elif k in ("norm", "norm_grad"):
        # activations: rows of different magnitude, off centre
        gen = _gen(seed, 2)
        wide = torch.randn((c["cap"], c["dim"] + c["spare"]), device=DEV, generator=gen)
        wide.mul_(torch.rand((c["cap"], 1), device=DEV, generator=gen).mul_(3).add_(0.2)).add_(torch.randn((c["cap"], 1), device=DEV, generator=gen))
        x = wide.to(DTYPES[c["x"]])[:, :c["dim"]]
        w = torch.randn(c["dim"], device=DEV, generator=gen).mul_(0.1).add_(1).to(DTYPES[c["par"]])
        s.update(x=x, n=_count(c["rows"]), w=w)
        if k == "norm":
            s.update(b=_randn((c["dim"],), c["par"], gen, 0.1), y=torch.zeros((c["cap"], c["dim"]), dtype=x.dtype, device=DEV),
                     mean=torch.zeros(c["cap"], device=DEV), rstd=torch.zeros(c["cap"], device=DEV))
        else:
            v, m = torch.var_mean(x.float(), 1, correction=0)
            s.update(dy=_randn((c["cap"], c["dim"]), c["x"], gen, 0.01), mean=m, rstd=(v + EPS).rsqrt(),
                     dx=torch.zeros((c["cap"], c["dim"]), dtype=x.dtype, device=DEV), dw=torch.zeros_like(w), db=torch.zeros_like(w))
    else:
        # the tensors of a model, views of one buffer, as buckets of gradients are
        sizes = _sizes(c)
        g = torch.randn(c["total"], device=DEV, generator=_gen(seed, 2)).mul_(0.05 / c["scale"]).to(DTYPES[c["g"]])
        o = torch.zeros(c["total"], dtype=DTYPES[c["out"]], device=DEV)
        s.update(flat=g, grads=_views(g, sizes), out=o, outs=_views(o, sizes), norm=torch.zeros(1, device=DEV))
    return s


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2110_08450_amd import binding as smfg
    c, k = s["case"], s["case"]["kind"]
    if k == "embed":
        smfg.embedding(s["table"], s["ids"], s["n"], c["cap"], s["out"], scale=c["scale"])
        return {"out": s["out"]}
    if k == "embed_grad":
        if "ws" not in s:  # kept from step to step, as a training program does
            s["ws"] = smfg.embedding_grad_workspace(c["cap"], c["rows"], c["dim"])
        if c["form"] == "rows":
            smfg.embedding_grad_rows(s["ids"], s["n"], c["cap"], s["dy"], c["rows"], s["row_ids"], s["num"], s["grad"], s["ws"], scale=c["scale"])
            return {"rows": s["row_ids"], "num": s["num"], "grad": s["grad"]}
        smfg.embedding_grad(s["ids"], s["n"], c["cap"], s["dy"], s["grad"], s["ws"], scale=c["scale"], accumulate=c["form"] == "add")
        return {"grad": s["grad"]}
    if k == "norm":
        smfg.layer_norm(s["x"], s["n"], c["cap"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if k == "norm_grad":
        if "ws" not in s:
            s["ws"] = smfg.layer_norm_grad_workspace(c["cap"], c["dim"])
        smfg.layer_norm_grad(s["dy"], s["x"], s["n"], c["cap"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["ws"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if "list" not in s:  # the gradients' buffers stay where they are from step to step
        s["list"] = smfg.grad_list(s["grads"], s["outs"])
    smfg.clip_grad_norm(s["list"], c["max_norm"], s["norm"], scale=c["scale"])
    return {"out": s["out"], "norm": s["norm"]}


def _run_plain(s):
    c, k = s["case"], s["case"]["kind"]
    if k == "embed":
        n = c["ids"]
        ids = s["ids"][:n].long()
        ok = (ids >= 0) & (ids < c["rows"])
        s["out"][:n] = s["table"][ids.clamp(0, c["rows"] - 1)].float() * (ok.float() * c["scale"])[:, None]
        return {"out": s["out"]}
    if k == "embed_grad":
        n = c["ids"]
        ids = s["ids"][:n].long()
        dy = s["dy"][:n].float()
        if c["form"] == "rows":
            rows, at = torch.unique(torch.where((ids >= 0) & (ids < c["rows"]), ids, c["rows"]), return_inverse=True)
            sums = torch.zeros((rows.numel(), c["dim"]), device=DEV).index_add_(0, at, dy) * c["scale"]
            u = int((rows < c["rows"]).sum())
            s["row_ids"][:u] = rows[:u].int()
            s["grad"][:u] = sums[:u]
            s["num"].fill_(u)
            return {"rows": s["row_ids"], "num": s["num"], "grad": s["grad"]}
        at = torch.where((ids >= 0) & (ids < c["rows"]), ids, c["rows"])
        sums = torch.zeros((c["rows"] + 1, c["dim"]), device=DEV).index_add_(0, at, dy)[:-1] * c["scale"]
        s["grad"].copy_(sums + s["grad"] if c["form"] == "add" else sums)
        return {"grad": s["grad"]}
    n = c.get("rows")
    if k == "norm":
        x = s["x"][:n].float()
        m = x.mean(1, keepdim=True)
        d = x - m
        r = 1 / torch.sqrt((d * d).mean(1, keepdim=True) + EPS)
        s["y"][:n] = d * r * s["w"].float() + s["b"].float()
        s["mean"][:n] = m[:, 0]
        s["rstd"][:n] = r[:, 0]
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if k == "norm_grad":
        dy, r = s["dy"][:n].float(), s["rstd"][:n, None]
        h = (s["x"][:n].float() - s["mean"][:n, None]) * r
        g = dy * s["w"].float()
        s["dx"][:n] = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        s["dw"].copy_((dy * h).sum(0))
        s["db"].copy_(dy.sum(0))
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    g = torch.cat([t.float() for t in s["grads"]]) * c["scale"]
    norm = torch.sqrt((g * g).sum())
    torch.cat([(t * torch.clamp(c["max_norm"] / (norm + 1e-6), max=1.0)).to(s["out"].dtype) for t in torch.split(g, [t.numel() for t in s["grads"]])],
              out=s["out"])
    s["norm"][0] = norm
    return {"out": s["out"], "norm": s["norm"]}


# ---- what a pass cannot do without ---------------------------------------------------------------

def _distinct(c):
    """Expected number of distinct ids of a call."""
    n, t = c["rows"], c["ids"]
    if c["law"] == "uniform":
        return n * -math.expm1(-t / n)
    edge = np.unique(np.concatenate([np.arange(1, min(n, 512) + 1), np.geomspace(1, n + 1, 2000).astype(np.int64), [n + 1]])).astype(np.float64)
    p = np.log(edge[1:] / edge[:-1]) / math.log(n + 1) / np.diff(edge)
    return float(np.sum(np.diff(edge) * -np.expm1(-t * p)))


def work(case):
    c, k = case, case["kind"]
    if k == "clip":
        return {"bytes": c["total"] * (SIZE[c["g"]] + SIZE[c["out"]]), "flops": 4 * c["total"]}
    n, e = (c["ids"] if "ids" in c else c["rows"]), c["dim"]
    if k == "embed":
        return {"bytes": n * SIZE[c["id"]] + _distinct(c) * e * SIZE[c["table"]] + n * e * SIZE[c["out"]], "flops": n * e}
    if k == "embed_grad":
        u = _distinct(c)
        out = {"dense": c["rows"] * e * SIZE[c["grad"]], "add": 2 * u * e * SIZE[c["grad"]], "rows": u * (e * SIZE[c["grad"]] + 4)}[c["form"]]
        return {"bytes": n * SIZE[c["id"]] + n * e * SIZE[c["dy"]] + out, "flops": n * e}
    if k == "norm":
        return {"bytes": 2 * n * e * SIZE[c["x"]] + 8 * n + 2 * e * SIZE[c["par"]], "flops": 7 * n * e}
    return {"bytes": 3 * n * e * SIZE[c["x"]] + 8 * n + 3 * e * SIZE[c["par"]], "flops": 13 * n * e}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------

def exact(case, seed):
    c, k = case, case["kind"]
    s = prepare(case, seed)
    if k == "clip":
        g = s["flat"].double() * c["scale"]
        norm = torch.linalg.vector_norm(g)
        return {"out": g.mul_(min(1.0, c["max_norm"] / (float(norm) + 1e-6))), "norm": norm.reshape(1)}
    if k == "embed":
        out = torch.zeros((c["cap"], c["dim"]), dtype=torch.float64, device=DEV)
        live = torch.nonzero(s["ids"][:c["ids"]] >= 0)[:, 0]
        out[live] = torch.index_select(s["table"], 0, s["ids"][live]).double() * c["scale"]
        return {"out": out}
    if k == "embed_grad":
        live = torch.nonzero(s["ids"][:c["ids"]] >= 0)[:, 0]
        by_id = s["ids"][live].long()
        order = torch.argsort(by_id, stable=True)
        rows, lengths = torch.unique_consecutive(by_id[order], return_counts=True)
        dy = s["dy"][live[order]].double() * c["scale"]
        # sums of consecutive rows: a column block at a time, as differences of running sums would lose digits
        sums = torch.segment_reduce(dy, "sum", lengths=lengths, axis=0) if rows.numel() else dy
        if c["form"] == "rows":
            grad = torch.zeros((c["cap"], c["dim"]), dtype=torch.float64, device=DEV)
            grad[:rows.numel()] = sums
            return {"rows": None, "num": None, "grad": grad}
        grad = s["grad"].double() if c["form"] == "add" else torch.zeros((c["rows"], c["dim"]), dtype=torch.float64, device=DEV)
        grad[rows] += sums
        return {"grad": grad}
    n = c["rows"]
    x = s["x"][:n].double()
    if k == "norm":
        var, mean = torch.var_mean(x, 1, correction=0)
        r = torch.rsqrt(var + EPS)
        out = {"y": torch.zeros((c["cap"], c["dim"]), dtype=torch.float64, device=DEV), "mean": torch.zeros(c["cap"], dtype=torch.float64, device=DEV),
               "rstd": torch.zeros(c["cap"], dtype=torch.float64, device=DEV)}
        out["mean"][:n], out["rstd"][:n] = mean, r
        out["y"][:n] = torch.addcmul(s["b"].double(), (x - mean[:, None]) * r[:, None], s["w"].double())
        return out
    # the gradient as the product with the norm's own derivative, for the given statistics
    dy, r, m = s["dy"][:n].double(), s["rstd"][:n].double(), s["mean"][:n].double()
    xh = x.sub(m[:, None]).mul_(r[:, None])
    wdy = dy * s["w"].double()
    a, b = wdy.sum(1) / c["dim"], torch.linalg.vecdot(wdy, xh) / c["dim"]
    dx = torch.zeros((c["cap"], c["dim"]), dtype=torch.float64, device=DEV)
    dx[:n] = (wdy - a[:, None] - b[:, None] * xh).mul_(r[:, None])
    return {"dx": dx, "dw": torch.linalg.vecdot(dy, xh, dim=0), "db": dy.sum(0)}
