"""The end of a training step on the last pipeline stage, operator by operator, as measurable cases.

A case is one pass through one operator: the output projection with its softmax cross entropy (`head_loss`: the loss alone,
`head_step`: the loss with the gradients of hidden states and weight), the global gradient norm with clipping (`clip`) and
the optimizer's update (`adamw`).  `run` computes the operator in its plain form, elementary torch operations in fp32, or,
where `own` is true, through the library's entry points.

Fields: op        head_loss, head_step, clip, adamw
        dtype     head: type of hidden states and weight (the weight's gradient is fp32); clip: type of the gradients;
                  adamw: type of the parameters ("bf16" ones have an fp32 master copy), whose gradients are fp32
  head  hidden, vocab, tokens
        ignored    share of the tokens that do not count (padding, prompts): label -100
        weighted   the tokens' losses have an upstream gradient each, otherwise one for all
        accumulate the weight's gradient is added to what the buffer holds
  clip, adamw: the tensors are slices of one flat buffer
        layers, hidden, ffn   the nine parameters of that many decoder layers
        tensors, largest, shapes   or that many tensors of 1 to `largest` elements, odd sizes and places among them, drawn
                  from the seed `shapes`
  clip  copies    clipped copies are written; otherwise the norm and the factor alone
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
IGNORED = -100
MAX_NORM, LR, BETA1, BETA2, EPS, DECAY, STEP = 1.0, 3e-4, 0.9, 0.95, 1e-8, 0.1, 1000


def _head(name, op, dtype, hidden, vocab, tokens, ignored=0.0, weighted=False, accumulate=False):
    return {"name": name, "op": op, "dtype": dtype, "hidden": hidden, "vocab": vocab, "tokens": tokens, "ignored": ignored,
            "weighted": weighted, "accumulate": accumulate}


def _layers(name, op, dtype, layers, hidden, ffn, copies=True):
    c = {"name": name, "op": op, "dtype": dtype, "layers": layers, "hidden": hidden, "ffn": ffn, "tensors": 0, "largest": 0, "shapes": 0}
    return dict(c, copies=copies) if op == "clip" else c


def _mixed(name, op, dtype, tensors, largest, shapes, copies=True):
    c = {"name": name, "op": op, "dtype": dtype, "layers": 0, "hidden": 0, "ffn": 0, "tensors": tensors, "largest": largest, "shapes": shapes}
    return dict(c, copies=copies) if op == "clip" else c


def listed():
    return [
        # The repository's smallest layer with a character-level vocabulary, fp32: a functional test of a training loop.
        # Microseconds of arithmetic, launches count.
        _head("f32 tiny head step", "head_step", "f32", 256, 1000, 128),
        # fp32 at a size where arithmetic counts: the reference run that a bf16 run is compared with; odd vocabulary.
        _head("f32 hidden-1024 head step", "head_step", "f32", 1024, 8001, 700, ignored=0.1),
        # The loss of a single token: scoring as a model answers.  One read of the weight.
        _head("loss of one token", "head_loss", "bf16", 4096, 32000, 1),
        # Evaluation of a ragged batch under a large odd vocabulary: the loss alone.
        _head("loss of 333, large vocabulary", "head_loss", "bf16", 2048, 100003, 333, ignored=0.1),
        # A small research model, ragged tokens, odd vocabulary, a weight of its own for each token.
        _head("small ragged head step", "head_step", "bf16", 1024, 50001, 700, ignored=0.3, weighted=True),
        # The last stage of a 7B-class model: one micro-batch of 2048 tokens.
        _head("7B-class head step", "head_step", "bf16", 4096, 32000, 2048),
        # The last stage of a 140B-class model: one micro-batch of 4096 tokens, gradients summed over micro-batches.
        _head("140B-class head step", "head_step", "bf16", 12288, 32000, 4096, accumulate=True),
        # Gradients of the tiny 4-layer stage: 36 tensors, 3 MB, latency.
        _layers("tiny stage clip", "clip", "f32", 4, 256, 704),
        # Gradients of a 7B-class layer: memory bandwidth.
        _layers("7B-class layer clip", "clip", "f32", 1, 4096, 11008),
        # The norm alone, of many bf16 gradients of all sizes in all places (adapters, biases, embeddings).
        _mixed("norm of 150 bf16 tensors", "clip", "bf16", 150, 20000000, 7, copies=False),
        # Parameters of the tiny stage, fp32.
        _layers("tiny stage update", "adamw", "f32", 4, 256, 704),
        # Parameters of a 7B-class layer: bf16 with fp32 master copy and moments.
        _layers("7B-class layer update", "adamw", "bf16", 1, 4096, 11008),
    ]


# ---------------------------------------------------------------------------------------------------------------- sizes
def _sizes(c):
    """Elements of each tensor of a clip or adamw case, in the order of the flat buffer: matrices first, then norm gains."""
    if c["layers"]:
        h, f = c["hidden"], c["ffn"]
        return [h * h] * (4 * c["layers"]) + [h * f] * (3 * c["layers"]) + [h] * (2 * c["layers"])
    r = random.Random(c["shapes"])
    return [max(1, int(math.exp(r.uniform(0.0, math.log(c["largest"]))))) for _ in range(c["tensors"])]


def _decayed(c):
    """How many of the tensors, from the first on, have weight decay: the matrices, or all but every tenth of mixed ones."""
    return 7 * c["layers"] if c["layers"] else c["tensors"] - c["tensors"] // 10


def _counted(c):
    return c["tokens"] * (1.0 - c["ignored"])


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["op"].startswith("head"):
        t, h, v = c["tokens"], c["hidden"], c["vocab"]
        b, products = (t + v) * h * es + 12.0 * t, 1
        if c["op"] == "head_step":
            b += t * h * es + 4.0 * v * h * (2 if c["accumulate"] else 1) + (4.0 * t if c["weighted"] else 0.0)
            products = 3
        return {"bytes": b, "flops": 2.0 * products * _counted(c) * h * v}
    n = float(sum(_sizes(c)))
    if c["op"] == "clip":
        return {"bytes": n * es * (2 if c["copies"] else 1), "flops": 3.0 * n}
    return {"bytes": n * (28 + (2 if c["dtype"] == "bf16" else 0)), "flops": 15.0 * n}


# ---------------------------------------------------------------------------------------------------------------- draws
def draw(rng):
    def log(lo, hi):
        return math.exp(rng.uniform(math.log(lo), math.log(hi)))

    def size(lo, hi, of=1):
        n = max(lo, min(hi, int(round(log(lo, hi) / of)) * of))
        return n + of if n == 3072 else n

    every = [work(c) for c in listed()]
    while True:
        op = rng.choice(("head_step", "head_step", "head_loss", "clip", "adamw"))
        if op.startswith("head"):
            dtype = "f32" if rng.random() < 0.25 else "bf16"
            top = 12288 if dtype == "bf16" else 1024
            c = _head("", op, dtype, size(64, top, 64 if dtype == "bf16" else 8), size(100, 131072 if dtype == "bf16" else 20000),
                      size(1, 8192 if dtype == "bf16" else 1500), rng.choice((0.0, 0.0, 0.1, 0.5)), rng.random() < 0.3,
                      rng.random() < 0.4)
        else:
            dtype = rng.choice(("bf16", "f32"))
            copies = op == "adamw" or rng.random() < 0.6
            if rng.random() < 0.5:
                c = _layers("", op, dtype, size(1, 12), size(64, 4096, 64), size(64, 11008, 64), copies)
            else:
                c = _mixed("", op, dtype, size(1, 400), size(1000, 50000000), rng.randrange(1 << 20), copies)
        w = work(c)
        most = every[8] if op == "clip" else every[11] if op == "adamw" else every[1] if dtype == "f32" else every[6]
        if w["bytes"] > max(most["bytes"], 1e8) or w["flops"] > most["flops"]:
            continue
        if op.startswith("head") and 8 * c["vocab"] * (c["hidden"] + c["tokens"]) > 12e9:   # in 64 bits
            continue
        del c["name"]
        return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype, scale=1.0, mean=0.0):
    t = torch.empty(shape, dtype=torch.float32, device=DEVICE)
    t.normal_(mean, scale, generator=gen)
    return t.to(dtype)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    dt = TYPES[c["dtype"]]
    s = {"case": c}
    if c["op"].startswith("head"):
        t, h, v = c["tokens"], c["hidden"], c["vocab"]
        # Normed hidden states that lean towards the label's row of the weight, as those of a trained model do: logits of
        # deviation 1.5, labels some 4 above them.
        s["w"] = _normal(gen, (v, h), dt, 1.5 / math.sqrt(h))
        labels = torch.randint(0, v, (t,), device=DEVICE, generator=gen)
        s["x"] = (_normal(gen, (t, h), torch.float32) + 1.8 * s["w"][labels].float()).to(dt)
        out = torch.rand(t, device=DEVICE, generator=gen) < c["ignored"]
        s["labels"] = torch.where(out, torch.full_like(labels, IGNORED), labels)
        s["scale"] = 1.0 / max(1.0, round(_counted(c)))
        s["dloss"] = torch.rand(t, device=DEVICE, generator=gen) if c["weighted"] else None
        s["loss"] = torch.empty(t, device=DEVICE)
        if c["op"] == "head_step":
            s["dx"] = torch.empty(t, h, dtype=dt, device=DEVICE)
            s["dw"] = _normal(gen, (v, h), torch.float32, 1e-4) if c["accumulate"] else torch.empty(v, h, device=DEVICE)
        return s
    n = sum(_sizes(c))
    if c["op"] == "clip":
        s["grad"] = _normal(gen, (n,), dt, 1e-2)
        s["out"] = torch.empty_like(s["grad"]) if c["copies"] else None
        s["result"] = torch.empty(2, device=DEVICE)
        return s
    s["grad"] = _normal(gen, (n,), torch.float32, 1e-2)
    s["master"] = _normal(gen, (n,), torch.float32, 0.02)
    s["param"] = s["master"].to(dt) if dt != torch.float32 else None
    s["m"] = _normal(gen, (n,), torch.float32, 2e-3)
    s["v"] = _normal(gen, (n,), torch.float32, 1e-2).square_()
    s["factor"] = torch.full((1,), 0.37, device=DEVICE)
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _plain_head(s):
    c = s["case"]
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"]
    logits = x @ w.t()
    top = logits.amax(dim=1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(dim=1, keepdim=True)
    counts = labels >= 0
    at = labels.clamp(min=0)[:, None]
    loss = (torch.log(total) + top - logits.gather(1, at))[:, 0] * counts
    if c["op"] == "head_loss":
        return {"loss": loss}
    g = (s["scale"] * counts if s["dloss"] is None else s["scale"] * s["dloss"] * counts)[:, None]
    d = e * (g / total)
    d.scatter_add_(1, at, -g)
    dx = (d @ w).to(s["x"].dtype)
    dw = d.t() @ x
    return {"loss": loss, "dx": dx, "dw": s["dw"].add_(dw) if c["accumulate"] else dw}


def _plain_clip(s):
    g = s["grad"].float()
    norm = g.square().sum().sqrt()
    factor = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
    out = {"result": torch.stack((norm, factor))}
    return dict(out, grad=(g * factor).to(s["grad"].dtype)) if s["case"]["copies"] else out


def _plain_adamw(s):
    c = s["case"]
    n = sum(_sizes(c)[:_decayed(c)])
    g = s["grad"] * s["factor"]
    s["m"].mul_(BETA1).add_(g, alpha=1.0 - BETA1)
    s["v"].mul_(BETA2).add_(g * g, alpha=1.0 - BETA2)
    step = (s["m"] / (1.0 - BETA1 ** STEP)) / ((s["v"] / (1.0 - BETA2 ** STEP)).sqrt() + EPS)
    s["master"][:n].mul_(1.0 - LR * DECAY)
    s["master"].sub_(LR * step)
    out = {"master": s["master"], "m": s["m"], "v": s["v"]}
    return out if s["param"] is None else dict(out, param=s["param"].copy_(s["master"]))


# ------------------------------------------------------------------------------------------------- the library's kernels
_kept = {}   # what a program keeps: the context, one workspace


def _workspace(size):
    if _kept.get("size", -1) < size:
        _kept["ws"], _kept["size"] = torch.empty(size, dtype=torch.uint8, device=DEVICE), size
    return _kept["ws"]


def _slices(flat, sizes):
    return [None] * len(sizes) if flat is None else torch.split(flat, sizes)


def _own(s):
    from paper_2405_16256_amd import binding as hh
    c = s["case"]
    if "ctx" not in _kept:
        _kept["ctx"] = hh.hh_ctx_create(0)
    ctx, stream = _kept["ctx"], torch.cuda.current_stream().cuda_stream
    if c["op"].startswith("head"):
        if "cfg" not in s:
            s["cfg"] = hh.make_head_cfg(c["hidden"], c["vocab"], c["tokens"], hh.HH_BF16 if c["dtype"] == "bf16" else hh.HH_F32)
            s["sizes"] = hh.hh_head_sizes(s["cfg"])
        if c["op"] == "head_loss":
            hh.hh_head_loss(ctx, s["cfg"], s["x"], s["w"], s["labels"], s["loss"], _workspace(s["sizes"][0]), stream)
            return {"loss": s["loss"]}
        hh.hh_head_step(ctx, s["cfg"], s["x"], s["w"], s["labels"], s["dloss"], s["scale"], s["loss"], s["dx"], s["dw"],
                        c["accumulate"], _workspace(s["sizes"][1]), stream)
        return {"loss": s["loss"], "dx": s["dx"], "dw": s["dw"]}
    if c["op"] == "clip":
        if "list" not in s:
            z = _sizes(c)
            s["list"] = hh.make_clip_tensors(list(zip(_slices(s["grad"], z), _slices(s["out"], z))))
        hh.hh_grad_clip(ctx, s["list"], MAX_NORM, s["result"], _workspace(hh.HH_CLIP_WORKSPACE_BYTES), stream)
        return {"result": s["result"], "grad": s["out"]} if c["copies"] else {"result": s["result"]}
    if "list" not in s:
        z = _sizes(c)
        decay = [DECAY] * _decayed(c) + [0.0] * (len(z) - _decayed(c))
        flat = {k: _slices(s[k], z) for k in ("param", "master", "m", "v", "grad")}
        if s["param"] is None:   # an fp32 parameter is its own master copy
            flat["param"], flat["master"] = flat["master"], flat["param"]
        s["list"] = hh.make_adamw_tensors(list(zip(flat["param"], flat["master"], flat["m"], flat["v"], flat["grad"], decay)))
        s["hyper"] = hh.make_adamw_cfg(LR, BETA1, BETA2, EPS, STEP)
    hh.hh_adamw_step(ctx, s["hyper"], s["list"], s["factor"], stream)
    out = {"master": s["master"], "m": s["m"], "v": s["v"]}
    return out if s["param"] is None else dict(out, param=s["param"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_head(state) if op.startswith("head") else _plain_clip(state) if op == "clip" else _plain_adamw(state)


# -------------------------------------------------------------------------------------------------- definition, 64 bits
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "clip":
        g = s["grad"].double()
        norm = torch.linalg.vector_norm(g)
        factor = torch.clamp(MAX_NORM / (norm + 1e-6), max=1.0)
        out = {"result": torch.stack((norm, factor))}
        return dict(out, grad=g * factor) if c["copies"] else out
    if c["op"] == "adamw":
        g = s["grad"].double() * s["factor"].double()
        m, v, p = s["m"].double(), s["v"].double(), s["master"].double()
        m = BETA1 * m + (1.0 - BETA1) * g
        v = BETA2 * v + (1.0 - BETA2) * g ** 2
        decay = torch.zeros_like(p)
        decay[:sum(_sizes(c)[:_decayed(c)])] = DECAY
        p = p - LR * (m / (1.0 - BETA1 ** STEP) / (torch.sqrt(v / (1.0 - BETA2 ** STEP)) + EPS) + decay * p)
        out = {"master": p, "m": m, "v": v}
        return out if s["param"] is None else dict(out, param=p)
    x, w, labels = s["x"].double(), s["w"].double(), s["labels"]
    counts = torch.nonzero(labels != IGNORED)[:, 0]   # the tokens that count, and they alone
    logits = torch.matmul(x[counts], w.t())
    chosen = labels[counts]
    lse = torch.logsumexp(logits, dim=1)
    rows = torch.arange(len(counts), device=DEVICE)
    loss = torch.zeros(len(labels), dtype=torch.float64, device=DEVICE)
    loss[counts] = lse - logits[rows, chosen]
    if c["op"] == "head_loss":
        return {"loss": loss}
    up = torch.full_like(loss, s["scale"]) if s["dloss"] is None else s["scale"] * s["dloss"].double()
    p = logits.sub_(lse[:, None]).exp_()
    p[rows, chosen] -= 1.0
    p.mul_(up[counts][:, None])
    dx = torch.zeros(len(labels), w.shape[1], dtype=torch.float64, device=DEVICE)
    dx[counts] = torch.matmul(p, w)
    dw = torch.matmul(p.t(), x[counts])
    return {"loss": loss, "dx": dx, "dw": dw + s["dw"].double() if c["accumulate"] else dw}
