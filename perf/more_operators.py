"""Performance cases of further operators of a training step on one MI355X: root-mean-square norm with the residual's addition (plain
and 8-bit outputs) and its gradient, softmax cross entropy with its gradient, AdamW over many tensors and over touched rows.

A case is a dict of plain values.  Five kinds of work, each through the package's public calls:

  rms         rms_norm: total = x + residual, the norm of total, as x's type ("same") or in 8 bits with scales ("e4m3", "i8")
  rms_grad    rms_norm_grad: gradients of the total and of the weight
  loss        cross_entropy: mean loss of the counted rows, and the logits' gradient
  adamw       adamw over a list of tensors, states in 32 or in 8 bits; 8-bit states are read out by adamw_values
  adamw_rows  adamw over the touched rows of a table

As everywhere in the package, the number of rows in use lives on the device, and buffers have room for more.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn, "i8": torch.int8,
          "i32": torch.int32, "i64": torch.int64}
SIZE = {"f16": 2, "bf16": 2, "f32": 4, "e4m3": 1, "i8": 1, "i32": 4, "i64": 8}
TOP = {"e4m3": 448.0, "i8": 127.0}  # largest value of an 8-bit type
EPS = 1e-6
BLOCK = 128  # elements that share the scale of an 8-bit state
BETAS, ADAM_EPS, DECAY, LR = (0.9, 0.999), 1e-8, 0.01, 1e-3


def listed():
    return [
        # the norm between two layers while one token each of eight requests is answered: latency
        dict(name="rms_request", kind="rms", rows=8, cap=8, dim=4096, x="bf16", par="bf16", spare=0, res=True, out="same", group=0),
        # the norm between the first layers, with the skip connection, a row per node of the middle frontier
        dict(name="rms_hidden", kind="rms", rows=154_321, cap=180_224, dim=256, x="f16", par="f32", spare=0, res=True, out="same", group=0),
        # wide hidden states for a product in 8 bits, a scale for 128 columns
        dict(name="rms_bytes", kind="rms", rows=16_384, cap=16_384, dim=4096, x="bf16", par="bf16", spare=0, res=True, out="e4m3", group=128),
        # gradient over the raw features' odd width, rows in a wider buffer
        dict(name="rms_grad_odd", kind="rms_grad", rows=47_062, cap=50_000, dim=301, x="f32", par="f32", spare=19, res=False),
        # gradient of wide hidden states, that of the skip connection added
        dict(name="rms_grad_wide", kind="rms_grad", rows=16_384, cap=16_384, dim=4096, x="bf16", par="bf16", spare=0, res=True),
        # a row per seed, a class per label: latency
        dict(name="loss_seeds", kind="loss", rows=1024, cap=1024, classes=172, x="f16", label="i32", spare=0, scale=1024.0),
        # many nodes, an odd number of classes, rows in a wider buffer
        dict(name="loss_odd", kind="loss", rows=33_333, cap=36_000, classes=1013, x="f32", label="i64", spare=3, scale=1.0),
        # a token to predict from a large vocabulary
        dict(name="loss_tokens", kind="loss", rows=8192, cap=8192, classes=50_000, x="bf16", label="i64", spare=0, scale=1.0),
        # all parameters of a three-layer GraphSAGE: latency
        dict(name="adamw_sage", kind="adamw", tensors=9, total=280_748, p="f32", g="f32", copy="none", state="f32", align=1),
        # touched rows of learned node embeddings of a products-sized graph
        dict(name="adamw_edges", kind="adamw_rows", rows=2_450_000, dim=100, ids=240_000, cap=260_000, g="f32", state="f32"),
        # all parameters of a large model: float ones with half copies for the next step, half gradients, clipped by a norm that is at hand
        dict(name="adamw_large", kind="adamw", tensors=290, total=400_000_000, p="f32", g="f16", copy="f16", state="f32", align=128),
        # the same model where memory is short: parameters and gradients of 16 bits, states of 8
        dict(name="adamw_bytes", kind="adamw", tensors=290, total=400_000_000, p="bf16", g="bf16", copy="none", state="i8", align=128),
    ]


# ---- cases drawn from the same ranges ------------------------------------------------------------

def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def _dim(rng):
    return rng.choice([rng.randint(1, 700), 8 * rng.randint(1, 64), rng.choice([32, 100, 128, 172, 256]), 1024 * rng.choice([1, 2, 4, 5, 6, 8])])


def draw(rng):
    kind = rng.choice(["rms", "rms", "rms_grad", "loss", "loss", "adamw", "adamw", "adamw_rows"])
    x = rng.choice(["f16", "bf16", "f32"])
    while True:
        if kind in ("rms", "rms_grad"):
            dim = _dim(rng)
            n = _log(rng, 1, max(4, min(200_000, 67_000_000 // dim)))
            c = dict(kind=kind, rows=n, cap=n + rng.choice([0, 0, rng.randint(1, 1 + n // 4)]), dim=dim, x=x, par=rng.choice([x, "f32"]),
                     spare=rng.choice([0, 0, rng.randint(1, 64)]), res=rng.random() < 0.7)
            if kind == "rms":
                out = rng.choice(["same", "same", "e4m3", "i8"])
                c.update(out=out, group=0 if out == "same" else rng.choice([0, 32, 64, 128]))
            return c
        if kind == "loss":
            k = _log(rng, 2, 150_000)
            n = _log(rng, 1, max(4, min(200_000, 200_000_000 // k)))
            return dict(kind=kind, rows=n, cap=n + rng.choice([0, 0, rng.randint(1, 1 + n // 4)]), classes=k, x=x, label=rng.choice(["i32", "i64"]),
                        spare=rng.choice([0, 0, rng.randint(1, 64)]), scale=1.0 if x != "f16" else 1024.0)
        state = rng.choice(["f32", "i8"])
        if kind == "adamw_rows":
            dim = rng.choice([rng.randint(1, 300), 8 * rng.randint(1, 64)])
            rows = _log(rng, 100, min(3_000_000, 300_000_000 // dim))
            n = _log(rng, 1, max(4, min(rows // 4, 70_000_000 // dim)))
            c = dict(kind=kind, rows=rows, dim=dim, ids=n, cap=min(rows, n + rng.choice([0, rng.randint(1, 1 + n // 4)])), g=x, state=state)
        else:
            p = rng.choice(["f32", "f32", x])
            c = dict(kind=kind, tensors=_log(rng, 1, 400), total=_log(rng, 10_000, 300_000_000), p=p, g=rng.choice([p, "f16", "bf16"]) if p == "f32" else p,
                     copy=rng.choice(["none", "f16", "bf16"]) if p == "f32" else "none", state=state, align=128 if state == "i8" else rng.choice([1, 128]))
            if c["total"] < 512 * c["tensors"]:
                continue
        return c


# ---- inputs --------------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 16 + salt)


def _randn(shape, dtype, gen, mul=1.0):
    return torch.randn(shape, device=DEV, dtype=torch.float32, generator=gen).mul_(mul).to(DTYPES[dtype])


def _count(n):
    return torch.tensor([n], dtype=torch.int64, device=DEV)


def _rows(c, cols, gen):
    """Activations: rows of different magnitude, off centre, in a buffer with spare columns."""
    wide = torch.randn((c["cap"], cols + c["spare"]), device=DEV, generator=gen)
    wide.mul_(torch.rand((c["cap"], 1), device=DEV, generator=gen).mul_(3).add_(0.2)).add_(torch.randn((c["cap"], 1), device=DEV, generator=gen))
    return wide.to(DTYPES[c["x"]])[:, :cols]


def _groups(c):
    return -(-c["dim"] // (c["group"] or c["dim"]))


def _layout(c):
    """(length, place in a flat buffer) of the tensors of a model: matrices of a few sizes, each with a vector or two behind it, the first takes the
    rest; and the buffer's length."""
    n, total, align = c["tensors"], c["total"], c["align"]
    w = [(0.7, 0.003, 1.0, 0.002, 0.25)[i % 5] for i in range(n)]
    sizes = [max(1, int(total * x / sum(w)) - (i % 3)) for i, x in enumerate(w)]
    sizes[0] += total - sum(sizes)
    at, places = 0, []
    for s in sizes:
        places.append(at)
        at += -(-s // align) * align
    return sizes, places, at


def _views(flat, c):
    sizes, places, _ = _layout(c)
    return [flat[p:p + s] for s, p in zip(sizes, places)]


def _padding(buffers, c):
    """Zeros between the tensors of flat buffers, in place; a step leaves them zeros."""
    sizes, places, end = _layout(c)
    for s, p, q in zip(sizes, places, places[1:] + [end]):
        if p + s < q:
            for t in buffers:
                t[p + s:q] = 0


def _codes(m, u):
    """8-bit states of blocks (rows of m and of u, the second moment's roots), and their scales."""
    a, b = m.abs().amax(1, keepdim=True), u.amax(1, keepdim=True)
    cm = torch.where(a > 0, torch.round(127 * torch.sqrt(m.abs() / a)), 0.0) * torch.sign(m)
    cu = torch.where(u > 0, torch.round(255 * torch.sqrt(u / b)).clamp_(min=1), 0.0)
    return cm.to(torch.int8), a[:, 0].contiguous(), cu.to(torch.uint8), b[:, 0].contiguous()


def prepare(case, seed):
    c, k = case, case["kind"]
    s = {"case": c}
    gen = _gen(seed, 2)
    if k in ("rms", "rms_grad"):
        w = torch.randn(c["dim"], device=DEV, generator=gen).mul_(0.1).add_(1).to(DTYPES[c["par"]])
        x = _rows(c, c["dim"], gen)
        s.update(x=x, n=_count(c["rows"]), w=w)
        if k == "rms":
            s.update(res=_rows(c, c["dim"], gen) if c["res"] else None, total=torch.zeros((c["cap"], c["dim"]), dtype=x.dtype, device=DEV) if c["res"] else None)
            if c["out"] == "same":
                s.update(y=torch.zeros((c["cap"], c["dim"]), dtype=x.dtype, device=DEV), rstd=torch.zeros(c["cap"], device=DEV))
            else:
                s.update(y=torch.zeros((c["cap"], c["dim"]), device=DEV).to(DTYPES[c["out"]]), scales=torch.zeros((c["cap"], _groups(c)), device=DEV))
        else:
            s.update(dy=_randn((c["cap"], c["dim"]), c["x"], gen, 0.01), dtotal=_randn((c["cap"], c["dim"]), c["x"], gen, 0.01) if c["res"] else None,
                     rstd=(x.float().square().mean(1) + EPS).rsqrt(), dx=torch.zeros((c["cap"], c["dim"]), dtype=x.dtype, device=DEV), dw=torch.zeros_like(w))
    elif k == "loss":
        x = _rows(c, c["classes"], gen)
        y = torch.randint(0, c["classes"], (c["cap"],), device=DEV, generator=gen)
        y[torch.rand(c["cap"], device=DEV, generator=gen) < 0.05] = -100  # not to be learned from
        s.update(x=x, y=y.to(DTYPES[c["label"]]), n=_count(c["rows"]), loss=torch.zeros(1, device=DEV),
                 dx=torch.zeros((c["cap"], c["classes"]), dtype=x.dtype, device=DEV))
    elif k == "adamw":
        end = _layout(c)[2]
        p, g = _randn((end,), c["p"], gen, 0.02), _randn((end,), c["g"], gen, 0.003)
        m, u = torch.randn(end, device=DEV, generator=gen).mul_(0.001), torch.randn(end, device=DEV, generator=gen).mul_(0.003).abs_()
        _padding((p, g, m, u), c)
        norm = torch.linalg.vector_norm(g, dtype=torch.float32).reshape(1)
        s.update(p=p, g=g, norm=norm, max_norm=1.0, step=100,
                 copy=torch.zeros(end, dtype=DTYPES[c["copy"]], device=DEV) if c["copy"] != "none" else None)
        if c["state"] == "f32":
            s.update(m=m, v=u * u)
        else:
            cm, a, cu, b = _codes(m.reshape(-1, BLOCK), u.reshape(-1, BLOCK))
            s.update(m=cm.reshape(-1), v=cu.reshape(-1), ms=a, vs=b, mv=torch.zeros(end, dtype=torch.bfloat16, device=DEV),
                     vv=torch.zeros(end, dtype=torch.bfloat16, device=DEV))
    else:
        r, d = c["rows"], c["dim"]
        ids = torch.randperm(r, device=DEV, generator=gen)[:c["cap"]].sort().values.int()
        s.update(p=_randn((r, d), "f32", gen, 0.1), g=_randn((c["cap"], d), c["g"], gen, 0.003), ids=ids, n=_count(c["ids"]), step=7)
        m, u = torch.randn((r, d), device=DEV, generator=gen).mul_(0.001), torch.randn((r, d), device=DEV, generator=gen).mul_(0.003).abs_()
        if c["state"] == "f32":
            s.update(m=m, v=u * u)
        else:
            pad = -(-d // BLOCK) * BLOCK
            cm, a, cu, b = _codes(*[torch.nn.functional.pad(t, (0, pad - d)).reshape(-1, BLOCK) for t in (m, u)])
            s.update(m=cm.reshape(r, pad)[:, :d].contiguous(), v=cu.reshape(r, pad)[:, :d].contiguous(), ms=a.reshape(r, -1), vs=b.reshape(r, -1),
                     mv=torch.zeros((r, d), dtype=torch.bfloat16, device=DEV), vv=torch.zeros((r, d), dtype=torch.bfloat16, device=DEV))
    return s


# ---- one pass ------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2110_08450_amd import binding as smfg
    c, k = s["case"], s["case"]["kind"]
    if k == "rms":
        if c["out"] == "same":
            smfg.rms_norm(s["x"], s["n"], c["cap"], s["w"], EPS, s["y"], residual=s["res"], total=s["total"], rstd=s["rstd"])
            return {"y": s["y"], "total": s["total"], "rstd": s["rstd"]}
        smfg.rms_norm(s["x"], s["n"], c["cap"], s["w"], EPS, s["y"], residual=s["res"], total=s["total"], scales=s["scales"], group=c["group"])
        return {"y": s["y"] if c["out"] == "e4m3" else _values(c, s["y"], s["scales"]), "scales": s["scales"], "total": s["total"]}
    if k == "rms_grad":
        if "ws" not in s:  # kept from step to step, as a training program does
            s["ws"] = smfg.rms_norm_grad_workspace(c["cap"], c["dim"])
        smfg.rms_norm_grad(s["dy"], s["x"], s["n"], c["cap"], s["w"], s["rstd"], s["dx"], s["dw"], s["ws"], grad_total=s["dtotal"])
        return {"dx": s["dx"], "dw": s["dw"]}
    if k == "loss":
        if "ws" not in s:
            s["ws"] = smfg.cross_entropy_workspace(c["cap"], c["classes"])
        smfg.cross_entropy(s["x"], s["y"], s["n"], c["cap"], s["loss"], s["ws"], grad_logits=s["dx"], scale=c["scale"])
        return {"loss": s["loss"], "dx": s["dx"]}
    if k == "adamw":
        if "list" not in s:  # the buffers stay where they are from step to step
            views = [_views(s[t], c) for t in ("p", "g", "m", "v")]
            more = {"copies": _views(s["copy"], c)} if s["copy"] is not None else {}
            if c["state"] == "i8":
                sizes, places, _ = _layout(c)
                more.update({n: [s[t][p // BLOCK:p // BLOCK + -(-z // BLOCK)] for z, p in zip(sizes, places)] for n, t in (("m_scales", "ms"), ("v_scales", "vs"))})
            s["list"] = smfg.adamw_list(*views, weight_decay=DECAY, **more)
        s["step"] += 1
        smfg.adamw(s["list"], s["step"], LR, betas=BETAS, eps=ADAM_EPS, max_norm=s["max_norm"], norm=s["norm"])
        if c["state"] == "i8":
            smfg.adamw_values(s["m"], s["ms"], s["mv"])
            smfg.adamw_values(s["v"], s["vs"], s["vv"])
            return {"p": s["p"], "m": s["mv"], "v": s["vv"]}
        return {"p": s["p"], "m": s["m"], "v": s["v"], "copy": s["copy"]}
    if "list" not in s:
        scales = {"m_scales": [s["ms"]], "v_scales": [s["vs"]]} if c["state"] == "i8" else {}
        s["list"] = smfg.adamw_list([s["p"]], [s["g"]], [s["m"]], [s["v"]], rows=[s["n"]], row_ids=[s["ids"]], weight_decay=DECAY, **scales)
    s["step"] += 1
    smfg.adamw(s["list"], s["step"], LR, betas=BETAS, eps=ADAM_EPS)
    if c["state"] == "i8":
        smfg.adamw_values(s["m"], s["ms"], s["mv"])
        smfg.adamw_values(s["v"], s["vs"], s["vv"])
        return {"p": s["p"], "m": s["mv"], "v": s["vv"]}
    return {"p": s["p"], "m": s["m"], "v": s["v"]}


def _values(c, q, scales):
    """What whole numbers with scales stand for."""
    return (q.float() * torch.repeat_interleave(scales, c["group"] or c["dim"], 1)[:, :c["dim"]]).to(torch.bfloat16)


def _values_of_codes(cm, a, cu, b):
    x, u = cm.float() / 127, cu.float() / 255
    return a[..., None] * x * x.abs(), (b[..., None] * u * u).square()


def _moments(s, m, v, g):
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g * g
    s["step"] += 1
    step = LR / -math.expm1(s["step"] * math.log(BETAS[0]))
    root = math.sqrt(-math.expm1(s["step"] * math.log(BETAS[1])))
    return m, v, lambda p: p - LR * DECAY * p - step * m / (torch.sqrt(v) / root + ADAM_EPS)


def _run_plain(s):
    c, k = s["case"], s["case"]["kind"]
    n = c.get("rows")
    if k == "rms":
        h = s["x"][:n].float()
        if c["res"]:
            s["total"][:n] = h + s["res"][:n].float()
            h = s["total"][:n].float()  # the norm is of the sum as the next layer and the gradient read it
        r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
        y = h * r * s["w"].float()
        if c["out"] == "same":
            s["y"][:n] = y
            s["rstd"][:n] = r[:, 0]
            return {"y": s["y"], "total": s["total"], "rstd": s["rstd"]}
        width = c["group"] or c["dim"]
        y = torch.nn.functional.pad(y, (0, _groups(c) * width - c["dim"])).reshape(n, -1, width)
        top = y.abs().amax(2, keepdim=True)
        q = torch.where(top > 0, y * (TOP[c["out"]] / top), 0.0).reshape(n, -1)[:, :c["dim"]]
        s["y"][:n] = (torch.round(q) if c["out"] == "i8" else q).to(s["y"].dtype)
        s["scales"][:n] = top[:, :, 0] / TOP[c["out"]]
        return {"y": s["y"] if c["out"] == "e4m3" else _values(c, s["y"], s["scales"]), "scales": s["scales"], "total": s["total"]}
    if k == "rms_grad":
        dy, r = s["dy"][:n].float(), s["rstd"][:n, None]
        h = s["x"][:n].float() * r
        g = dy * s["w"].float()
        dx = r * (g - h * (g * h).mean(1, keepdim=True))
        s["dx"][:n] = dx + s["dtotal"][:n].float() if c["res"] else dx
        s["dw"].copy_((dy * h).sum(0))
        return {"dx": s["dx"], "dw": s["dw"]}
    if k == "loss":
        x, y = s["x"][:n].float(), s["y"][:n].long()
        ok = (y >= 0) & (y < c["classes"])
        at = torch.where(ok, y, 0)[:, None]
        x = x - x.amax(1, keepdim=True)
        e = torch.exp(x)
        total = e.sum(1, keepdim=True)
        many = ok.sum().clamp(min=1)
        s["loss"][0] = torch.where(ok, torch.log(total[:, 0]) - x.gather(1, at)[:, 0], 0.0).sum() / many
        p = e / total
        p.scatter_add_(1, at, torch.full_like(total, -1.0))
        s["dx"][:n] = p * torch.where(ok, c["scale"] / many, 0.0)[:, None]
        return {"loss": s["loss"], "dx": s["dx"]}
    if k == "adamw":
        g = s["g"].float() * torch.clamp(s["max_norm"] / (s["norm"] + 1e-6), max=1.0)
        if c["state"] == "f32":
            m, v, update = _moments(s, s["m"], s["v"], g)
            s["m"].copy_(m), s["v"].copy_(v)
        else:
            m, v = _values_of_codes(s["m"].reshape(-1, BLOCK), s["ms"], s["v"].reshape(-1, BLOCK), s["vs"])
            m, v, update = _moments(s, m.reshape(-1), v.reshape(-1), g)
        p = update(s["p"].float())
        s["p"].copy_(p)
        if c["state"] == "i8":
            cm, a, cu, b = _codes(m.reshape(-1, BLOCK), torch.sqrt(v).reshape(-1, BLOCK))
            s["m"].copy_(cm.reshape(-1)), s["ms"].copy_(a), s["v"].copy_(cu.reshape(-1)), s["vs"].copy_(b)
            m, v = _values_of_codes(cm, a, cu, b)
            s["mv"].copy_(m.reshape(-1)), s["vv"].copy_(v.reshape(-1))
            return {"p": s["p"], "m": s["mv"], "v": s["vv"]}
        if s["copy"] is not None:
            s["copy"].copy_(p)
        return {"p": s["p"], "m": s["m"], "v": s["v"], "copy": s["copy"]}
    n, d = c["ids"], c["dim"]
    ids, g = s["ids"][:n].long(), s["g"][:n].float()
    if c["state"] == "f32":
        m, v, update = _moments(s, s["m"][ids], s["v"][ids], g)
        s["m"][ids], s["v"][ids] = m, v
        s["p"][ids] = update(s["p"][ids])
        return {"p": s["p"], "m": s["m"], "v": s["v"]}
    pad = -(-d // BLOCK) * BLOCK

    def blocks(t):
        return torch.nn.functional.pad(t, (0, pad - d)).reshape(t.shape[0], -1, BLOCK)

    def whole(t):
        return t.reshape(t.shape[0], pad)[:, :d]

    m, v = _values_of_codes(blocks(s["m"][ids]), s["ms"][ids], blocks(s["v"][ids]), s["vs"][ids])
    m, v, update = _moments(s, whole(m), whole(v), g)
    s["p"][ids] = update(s["p"][ids])
    cm, a, cu, b = _codes(blocks(m).reshape(-1, BLOCK), torch.sqrt(blocks(v)).reshape(-1, BLOCK))
    s["m"][ids], s["ms"][ids] = whole(cm.reshape(n, -1)), a.reshape(n, -1)
    s["v"][ids], s["vs"][ids] = whole(cu.reshape(n, -1)), b.reshape(n, -1)
    m, v = _values_of_codes(blocks(s["m"]), s["ms"], blocks(s["v"]), s["vs"])
    s["mv"].copy_(whole(m)), s["vv"].copy_(whole(v))
    return {"p": s["p"], "m": s["mv"], "v": s["vv"]}


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    c, k = case, case["kind"]
    if k in ("rms", "rms_grad"):
        n, e, x, p = c["rows"], c["dim"], SIZE[c["x"]], SIZE[c["par"]]
        if k == "rms_grad":
            return {"bytes": (4 if c["res"] else 3) * n * e * x + 4 * n + 2 * e * p, "flops": 11 * n * e}
        out = n * e * x + 4 * n if c["out"] == "same" else n * e + 4 * n * _groups(c)
        return {"bytes": (3 if c["res"] else 1) * n * e * x + out + e * p, "flops": 6 * n * e}
    if k == "loss":
        n, e = c["rows"], c["classes"]
        return {"bytes": 2 * n * e * SIZE[c["x"]] + n * SIZE[c["label"]], "flops": 8 * n * e}
    if k == "adamw":
        n = c["total"]
        each = 2 * SIZE[c["p"]] + SIZE[c["g"]] + (SIZE[c["copy"]] if c["copy"] != "none" else 0)
        each += 16 if c["state"] == "f32" else 4 + 16 / BLOCK + 4  # codes, scales, the values read out
        return {"bytes": n * each, "flops": 15 * n}
    n = c["ids"] * c["dim"]
    if c["state"] == "f32":
        return {"bytes": n * (24 + SIZE[c["g"]]) + 4 * c["ids"], "flops": 15 * n}
    return {"bytes": n * (12 + SIZE[c["g"]]) + (4 + 16 * -(-c["dim"] // BLOCK)) * c["ids"] + 6 * c["rows"] * c["dim"], "flops": 15 * n}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------

def _f64(*shape):
    return torch.zeros(shape, dtype=torch.float64, device=DEV)


def _exact_moments(p, m, v, g, t):
    m = torch.lerp(g, m, BETAS[0])
    v = torch.lerp(g.square(), v, BETAS[1])
    p = p * (1 - LR * DECAY) - LR * (m / (1 - BETAS[0] ** t)) / ((v / (1 - BETAS[1] ** t)).sqrt() + ADAM_EPS)
    return p, m, v


def _exact_states(cm, a, cu, b):
    cm, cu, a, b = cm.double(), cu.double(), a.double()[..., None], b.double()[..., None]
    return a * cm.sign() * (cm / 127).square(), b.square() * (cu / 255) ** 4


def _exact_stored(m, v):
    """What is left of states (blocks in the last dimension) that are held in 8 bits."""
    a = m.abs().amax(-1, keepdim=True)
    cm = ((m.abs() / a).nan_to_num(0.0).sqrt() * 127).round()
    b = v.amax(-1, keepdim=True)
    cu = ((v / b).nan_to_num(0.0) ** 0.25 * 255).round()
    cu = torch.maximum(cu, (v > 0).double())
    return m.sign() * a * (cm / 127) ** 2, b * (cu / 255) ** 4


def exact(case, seed):
    c, k = case, case["kind"]
    s = prepare(case, seed)
    n = c.get("rows")
    if k == "rms":
        h = s["x"][:n].double()
        out = {"total": None}
        if c["res"]:
            h = h + s["res"][:n].double()
            out["total"] = _f64(c["cap"], c["dim"])
            out["total"][:n] = h
            h = out["total"][:n].to(s["x"].dtype).double()
        r = 1 / (torch.linalg.vector_norm(h, dim=1).square() / c["dim"] + EPS).sqrt()
        y = h.mul_(r[:, None]).mul_(s["w"].double())
        if c["out"] == "same":
            out.update(y=_f64(c["cap"], c["dim"]), rstd=_f64(c["cap"]))
            out["y"][:n], out["rstd"][:n] = y, r
            return out
        width = c["group"] or c["dim"]
        out.update(scales=_f64(c["cap"], _groups(c)), y=_f64(c["cap"], c["dim"]))
        which = torch.arange(c["dim"], device=DEV) // width
        wide = _f64(n, _groups(c) * width)
        wide[:, :c["dim"]] = y.abs()
        out["scales"][:n] = wide.view(n, -1, width).amax(2) / TOP[c["out"]]
        q = (y / out["scales"][:n][:, which]).nan_to_num(0.0)
        if c["out"] == "i8":
            out["y"][:n] = q.round() * out["scales"][:n][:, which]
        else:  # three digits behind the first down to 2^-6, a fixed step of 2^-9 below
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            out["y"][:n] = (q / step).round() * step
        return out
    if k == "rms_grad":
        # the gradient as the product with the norm's own derivative, for the given statistics
        dy, r, x = s["dy"][:n].double(), s["rstd"][:n].double(), s["x"][:n].double()
        wdy = dy * s["w"].double()
        dot = torch.linalg.vecdot(wdy, x) * r ** 3 / c["dim"]
        dx = _f64(c["cap"], c["dim"])
        dx[:n] = wdy * r[:, None] - x * dot[:, None]
        if c["res"]:
            dx[:n] += s["dtotal"][:n].double()
        return {"dx": dx, "dw": torch.linalg.vecdot(dy, x * r[:, None], dim=0)}
    if k == "loss":
        x, y = s["x"][:n].double(), s["y"][:n].long()
        live = torch.nonzero(y >= 0)[:, 0]
        x, y = x[live], y[live]
        rows = torch.arange(live.numel(), device=DEV)
        lse = torch.logsumexp(x, 1)
        many = max(1, live.numel())
        loss = (lse - x[rows, y]).sum() / many
        p = x.sub_(lse[:, None]).exp_()
        p[rows, y] -= 1
        dx = _f64(c["cap"], c["classes"])
        dx[live] = p.mul_(c["scale"] / many)
        return {"loss": loss.reshape(1), "dx": dx}
    t = s["step"] + 1
    if k == "adamw":
        g = s["g"].double() * min(1.0, s["max_norm"] / (float(s["norm"]) + 1e-6))
        if c["state"] == "f32":
            m, v = s["m"].double(), s["v"].double()
        else:
            m, v = [x.reshape(-1) for x in _exact_states(s["m"].reshape(-1, BLOCK), s["ms"], s["v"].reshape(-1, BLOCK), s["vs"])]
        p, m, v = _exact_moments(s["p"].double(), m, v, g, t)
        out = {"p": p}
        if c["state"] == "i8":
            out["m"], out["v"] = [x.reshape(-1) for x in _exact_stored(m.reshape(-1, BLOCK), v.reshape(-1, BLOCK))]
        else:
            out.update(m=m, v=v, copy=None if s["copy"] is None else p)
        return out
    ids, d = s["ids"][:c["ids"]].long(), c["dim"]
    g = s["g"][:c["ids"]].double()
    if c["state"] == "f32":
        p, m, v = s["p"].double(), s["m"].double(), s["v"].double()
        p[ids], m[ids], v[ids] = _exact_moments(p[ids], m[ids], v[ids], g, t)
        return {"p": p, "m": m, "v": v}
    pad = -(-d // BLOCK) * BLOCK

    def blocks(x):
        wide = x.new_zeros((x.shape[0], pad))
        wide[:, :d] = x
        return wide.reshape(x.shape[0], -1, BLOCK)

    m, v = [x.reshape(c["rows"], pad)[:, :d].contiguous() for x in _exact_states(blocks(s["m"]), s["ms"], blocks(s["v"]), s["vs"])]
    p = s["p"].double()
    p[ids], new_m, new_v = _exact_moments(p[ids], m[ids], v[ids], g, t)
    m[ids], v[ids] = [x.reshape(c["ids"], pad)[:, :d] for x in _exact_stored(blocks(new_m), blocks(new_v))]
    return {"p": p, "m": m, "v": v}
