"""The residual path of a layer and products in microscaled 8- and 4-bit floating point, operator by operator, as measurable cases.

A case is one pass through one operator: dropout from a counter-based generator (`dropout`), the residual's addition of a dropped
branch with the root-mean-square norm behind it (`norm`) and its gradients (`norm_grad`), quantisation to blocks of 32 values
with a common scale (`quantise`) and the product of two such operands (`product`).  `run` computes the operator in its plain form,
elementary torch operations in fp32, or, where `own` is true, through the library's entry points.

Formats: "e4m3" and "e2m1" elements, each block of 32 along the contraction axis with a power of two as its scale.  In memory a row of
k values is padded with zeros to a multiple of 256; e4m3 takes a byte a value, e2m1 half of one (the even value in the low bits),
and a row's scales, a byte each (exponent + 127), are a row of their own.  What is held so is returned as the values it stands for, in bf16, which
holds them exactly.

Fields: op        dropout, norm, norm_grad, quantise, product
        dtype     of the tensors that are not packed ("bf16", "f32"); product: of the result
        rows, cols
  dropout, norm, norm_grad
        p         share of the values that are dropped (a multiple of 2^-16)
  norm, norm_grad
        branch    there is a branch to be dropped and added; otherwise the norm of x alone
  norm  format    of the packed copy of the normed rows ("none": there is none)
        normed    the normed rows are written unpacked
  norm_grad
        residual  a gradient reaches the sum from elsewhere too
        accumulate the gain's gradient is added to what the buffer holds
  quantise
        format, by ("row": blocks along a row, "column": the transposed copy with blocks along a column, "both")
  product   result [rows, cols] = a [rows, inner] b [cols, inner]^T
        inner, a, b (formats), accumulate
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5
BLOCK, PAD = 32, 256
TOP = {"e2m1": 2, "e4m3": 8}            # exponent of a format's largest value
LEAST = {"e2m1": 0, "e4m3": -6}         # exponent of its least normal value
FRACTION = {"e2m1": 1, "e4m3": 3}       # bits behind the point
LARGEST = {"e2m1": 6.0, "e4m3": 448.0}
BITS = {"e2m1": 4, "e4m3": 8}


def _dropout(name, dtype, rows, cols, p):
    return {"name": name, "op": "dropout", "dtype": dtype, "rows": rows, "cols": cols, "p": p}


def _norm(name, dtype, rows, cols, branch, p, format, normed):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "cols": cols, "branch": branch, "p": p, "format": format, "normed": normed}


def _norm_grad(name, dtype, rows, cols, branch, p, residual, accumulate):
    return {"name": name, "op": "norm_grad", "dtype": dtype, "rows": rows, "cols": cols, "branch": branch, "p": p, "residual": residual,
            "accumulate": accumulate}


def _quantise(name, dtype, rows, cols, format, by):
    return {"name": name, "op": "quantise", "dtype": dtype, "rows": rows, "cols": cols, "format": format, "by": by}


def _product(name, dtype, rows, cols, inner, a, b, accumulate=False):
    return {"name": name, "op": "product", "dtype": dtype, "rows": rows, "cols": cols, "inner": inner, "a": a, "b": b, "accumulate": accumulate}


def listed():
    return [
        # The repository's smallest layer, fp32: a functional test of a training loop.  Launches count.
        _dropout("dropout, tiny f32", "f32", 128, 256, 0.125),
        # A branch of a 140B-class layer, one micro-batch of 4096 tokens: memory bandwidth, and the generator's arithmetic.
        _dropout("dropout, 140B-class", "bf16", 4096, 12288, 0.09375),
        # One token of a 7B-class layer as a model answers: the row goes straight into an 8-bit product.
        _norm("norm of one token to e4m3", "bf16", 1, 4096, True, 0.0, "e4m3", False),
        # Odd rows and an odd width, fp32, as a reference run has it.
        _norm("norm, ragged f32", "f32", 700, 1003, True, 0.25, "none", True),
        # A residual connection of a 140B-class layer in training: dropout, sum, norm, kept in bf16 and packed for the product.
        _norm("norm to e4m3, 140B-class", "bf16", 4096, 12288, True, 0.09375, "e4m3", True),
        # The gradients of the ragged one.
        _norm_grad("norm gradients, ragged f32", "f32", 700, 1003, True, 0.25, True, True),
        # The gradients of the 140B-class one: two gradients in, two out, the gain's over all tokens.
        _norm_grad("norm gradients, 140B-class", "bf16", 4096, 12288, True, 0.09375, True, False),
        # Activations of a ragged batch, blocks along the rows.
        _quantise("quantise ragged rows to e4m3", "bf16", 333, 2050, "e4m3", "row"),
        # A 7B-class up projection, both ways round as training wants it: for the output and for the input's gradient.
        _quantise("quantise a 7B-class weight to e2m1", "bf16", 11008, 4096, "e2m1", "both"),
        # One token through a 7B-class down projection of 4-bit weights: a read of the weight.
        _product("product of one token, 7B-class", "bf16", 1, 4096, 11008, "e4m3", "e2m1"),
        # A small model's weight gradient, ragged in every direction, summed over micro-batches.
        _product("ragged e4m3 product, f32 sums", "f32", 1003, 700, 2050, "e4m3", "e4m3", True),
        # The gate and up projections of a 140B-class layer's share, all in 4 bits: the matrix cores.
        _product("e2m1 product, 140B-class", "bf16", 4096, 8192, 12288, "e2m1", "e2m1"),
    ]


# ---------------------------------------------------------------------------------------------------------------- sizes
def _es(c):
    return 2 if c["dtype"] == "bf16" else 4


def _packed(format):
    """Bytes a value, with its share of the scale."""
    return BITS[format] / 8.0 + 1.0 / BLOCK


def work(case):
    c = case
    n = float(c["rows"]) * c["cols"]
    if c["op"] == "dropout":
        return {"bytes": 2 * n * _es(c), "flops": 2 * n}
    if c["op"] == "norm":   # x, branch, sum, normed, packed and the values that this stands for
        tensors = 1 + 2 * c["branch"] + c["normed"]
        return {"bytes": n * (tensors * _es(c) + (_packed(c["format"]) + 2 if c["format"] != "none" else 0)), "flops": 8 * n}
    if c["op"] == "norm_grad":   # sum, gradient of the normed, of the sum; out: of x, of the branch
        return {"bytes": n * _es(c) * (3 + c["residual"] + c["branch"]), "flops": 14 * n}
    if c["op"] == "quantise":
        return {"bytes": n * (_es(c) + (2 if c["by"] == "both" else 1) * (_packed(c["format"]) + 2)), "flops": 6 * n}
    k = float(c["inner"])
    return {"bytes": k * (c["rows"] * _packed(c["a"]) + c["cols"] * _packed(c["b"])) + n * _es(c) * (1 + c["accumulate"]), "flops": 2 * n * k}


# ---------------------------------------------------------------------------------------------------------------- draws
def draw(rng):
    def size(lo, hi):
        n = math.exp(rng.uniform(math.log(lo), math.log(hi)))
        of = rng.choice((1, 1, 8, 64, 256))   # odd sizes, and those of models
        return max(lo, min(hi, int(round(n / of)) * of))

    most = {op: max(work(c)["bytes"] for c in listed() if c["op"] == op) for op in ("dropout", "norm", "norm_grad", "quantise")}
    flops = max(work(c)["flops"] for c in listed())
    while True:
        op = rng.choice(("dropout", "norm", "norm_grad", "quantise", "product", "product"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        p = rng.choice((0.0, 0.0625, 0.125, 0.25, 0.5))
        rows, cols = size(1, 8192), size(8, 16384)
        if op == "dropout":
            c = _dropout("", dtype, rows, cols, rng.choice((0.0625, 0.125, 0.25, 0.5)))
        elif op == "norm":
            branch, format = rng.random() < 0.7, rng.choice(("none", "e4m3", "e2m1"))
            c = _norm("", dtype, rows, cols, branch, p if branch else 0.0, format, format == "none" or rng.random() < 0.5)
        elif op == "norm_grad":
            branch = rng.random() < 0.7
            c = _norm_grad("", dtype, rows, cols, branch, p if branch else 0.0, rng.random() < 0.7, rng.random() < 0.4)
        elif op == "quantise":
            c = _quantise("", dtype, rows, cols, rng.choice(("e4m3", "e2m1")), rng.choice(("row", "column", "both")))
        else:
            c = _product("", dtype, rows, size(64, 16384), size(32, 16384), rng.choice(("e4m3", "e2m1")), rng.choice(("e4m3", "e2m1")),
                         dtype == "f32" and rng.random() < 0.4)
        w = work(c)
        if w["flops"] > flops or (op != "product" and w["bytes"] > most[op]):
            continue
        del c["name"]
        return c


# --------------------------------------------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype, scale=1.0, mean=0.0):
    t = torch.empty(shape, dtype=torch.float32, device=DEVICE)
    t.normal_(mean, scale, generator=gen)
    return t.to(dtype)


def _activations(gen, rows, cols, dtype):
    """Normal values with a few columns that are ten times as large, as hidden states have them."""
    t = _normal(gen, (rows, cols), torch.float32)
    big = torch.rand(cols, device=DEVICE, generator=gen) < 0.01
    return (t * (1.0 + 9.0 * big)).to(dtype)


def _pack(x, format):
    """Codes and scales of x as they lie in memory."""
    rows, cols = x.shape
    width = -(-cols // PAD) * PAD
    p, e = _blocks(x, format)
    if format == "e4m3":
        codes = p.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        steps = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEVICE)   # exact numbers of the format
        codes = (torch.bucketize(p.abs(), steps) + 8 * torch.signbit(p)).to(torch.uint8)
    codes, e = codes.reshape(rows, -1), e.reshape(rows, -1)
    full = torch.zeros(rows, width, dtype=torch.uint8, device=DEVICE)
    full[:, :codes.shape[1]] = codes
    scales = torch.zeros(rows, width // BLOCK, dtype=torch.uint8, device=DEVICE)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    if format == "e2m1":
        full = full[:, 0::2] | (full[:, 1::2] << 4)
    return full.contiguous(), scales


def _room(rows, cols, format):
    """Buffers that a packed tensor is written into."""
    width = -(-cols // PAD) * PAD
    return (torch.empty(rows, width * BITS[format] // 8, dtype=torch.uint8, device=DEVICE),
            torch.empty(rows, width // BLOCK, dtype=torch.uint8, device=DEVICE))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    dt, rows, cols = TYPES[c["dtype"]], c["rows"], c["cols"]
    s = {"case": c, "seed": (int(seed) * 0x9E3779B97F4A7C15 + 0x1234567) % 2 ** 63, "offset": int(seed) % 1000 + (5 << 32)}
    if c["op"] == "product":
        s["a"] = _pack(_activations(gen, rows, c["inner"], torch.float32), c["a"])
        s["b"] = _pack(_normal(gen, (cols, c["inner"]), torch.float32, 0.02), c["b"])
        s["out"] = _normal(gen, (rows, cols), dt, 0.1) if c["accumulate"] else torch.empty(rows, cols, dtype=dt, device=DEVICE)
        return s
    s["x"] = _activations(gen, rows, cols, dt)
    if c["op"] == "dropout":
        s["y"] = torch.empty_like(s["x"])
        return s
    if c["op"] == "quantise":
        if c["by"] != "column":
            s["by_row"], s["rows"] = _room(rows, cols, c["format"]), torch.empty(rows, cols, dtype=torch.bfloat16, device=DEVICE)
        if c["by"] != "row":
            s["by_column"], s["columns"] = _room(cols, rows, c["format"]), torch.empty(cols, rows, dtype=torch.bfloat16, device=DEVICE)
        return s
    s["g"] = _normal(gen, (cols,), dt, 0.1, 1.0)
    if c["op"] == "norm":
        s["branch"] = _normal(gen, (rows, cols), dt, 0.5) if c["branch"] else None
        s["sum"] = torch.empty_like(s["x"]) if c["branch"] else None
        s["normed"] = torch.empty_like(s["x"]) if c["normed"] else None
        if c["format"] != "none":
            s["packed"], s["values"] = _room(rows, cols, c["format"]), torch.empty(rows, cols, dtype=torch.bfloat16, device=DEVICE)
        return s
    s["dnormed"] = _normal(gen, (rows, cols), dt)
    s["dsum"] = _normal(gen, (rows, cols), dt) if c["residual"] else None
    s["dx"] = torch.empty_like(s["x"])
    s["dbranch"] = torch.empty_like(s["x"]) if c["branch"] else None
    s["dg"] = _normal(gen, (cols,), torch.float32) if c["accumulate"] else torch.empty(cols, device=DEVICE)
    return s


# ----------------------------------------------------------------------------------------------------------- plain form
def _factor(s):
    """What each value of a branch is multiplied by: 0 or one over the share that is kept.  Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
    "Parallel random numbers: as easy as 1, 2, 3", 2011) of (column / 8, row, offset) under the seed; eight values to a counter,
    16 bits each."""
    c = s["case"]
    rows, cols, dropped = c["rows"], c["cols"], round(c["p"] * 65536)
    if dropped == 0:
        return torch.ones((), device=DEVICE)
    low = 0xFFFFFFFF
    group = torch.arange((cols + 7) // 8, device=DEVICE)[None, :]
    row = torch.arange(rows, device=DEVICE)[:, None]
    w = (group, row, torch.full_like(row, s["offset"] & low), torch.full_like(row, s["offset"] >> 32))
    k0, k1 = s["seed"] & low, s["seed"] >> 32
    for _ in range(10):   # the generator's rounds, each of the one before
        a, b = w[0] * 0xD2511F53, w[2] * 0xCD9E8D57   # modulo 2^64, whose upper half is taken without the sign
        w = ((b >> 32 & low) ^ w[1] ^ k0, b & low, (a >> 32 & low) ^ w[3] ^ k1, a & low)
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    words = torch.stack(torch.broadcast_tensors(*w), dim=2)
    bits = torch.stack((words & 0xFFFF, words >> 16), dim=3).reshape(rows, -1)[:, :cols]
    return (bits >= dropped).float() * (65536.0 / (65536 - dropped))


def _blocks(x, format):
    """Numbers of the format and, a block of 32 each, the exponent of their scale; [rows, blocks, 32] and [rows, blocks, 1]."""
    x = x.float()
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % BLOCK)).reshape(rows, -1, BLOCK)
    most = x.abs().amax(dim=2, keepdim=True)
    e = torch.where(most > 0, torch.frexp(most).exponent - 1 - TOP[format], -127).clamp(min=-127)
    x = x * torch.exp2(-e.double()).float()
    step = torch.exp2((torch.frexp(x).exponent - 1).clamp(min=LEAST[format]).double() - FRACTION[format]).float()
    return (torch.round(x / step) * step).clamp(-LARGEST[format], LARGEST[format]), e


def _rounded(x, format):
    """The values that a packed copy of x stands for."""
    p, e = _blocks(x, format)
    return (p * torch.exp2(e.double()).float()).reshape(x.shape[0], -1)[:, :x.shape[1]].to(torch.bfloat16)


def _unpacked(codes, scales, cols, format):
    """The values of a packed tensor, fp32."""
    code = (torch.stack((codes & 15, codes >> 4), dim=2).reshape(codes.shape[0], -1) if format == "e2m1" else codes).int()
    f = FRACTION[format]
    sign = 1.0 - 2.0 * (code >> (BITS[format] - 1))
    code = code & ((1 << (BITS[format] - 1)) - 1)
    e, m = code >> f, (code & ((1 << f) - 1)).float() / (1 << f)
    value = sign * torch.where(e > 0, 1.0 + m, m) * torch.exp2((e.clamp(min=1) + LEAST[format] - 1).float())
    return (value.reshape(value.shape[0], -1, BLOCK) * torch.exp2(scales.float() - 127.0)[:, :, None]).reshape(value.shape)[:, :cols]


def _plain(s):
    c = s["case"]
    if c["op"] == "dropout":
        return {"y": (s["x"].float() * _factor(s)).to(s["x"].dtype)}
    if c["op"] == "quantise":
        rows = {"rows": _rounded(s["x"], c["format"])} if c["by"] != "column" else {}
        return dict(rows, columns=_rounded(s["x"].t(), c["format"])) if c["by"] != "row" else rows
    if c["op"] == "product":
        y = _unpacked(*s["a"], c["inner"], c["a"]) @ _unpacked(*s["b"], c["inner"], c["b"]).t()
        return {"out": s["out"].add_(y) if c["accumulate"] else y.to(s["out"].dtype)}
    dt, g = s["x"].dtype, s["g"].float()
    if c["op"] == "norm":
        out = {}
        h = s["x"].float()
        if c["branch"]:
            out["sum"] = (h + s["branch"].float() * _factor(s)).to(dt)
            h = out["sum"].float()   # the norm is of the sum as it is kept
        n = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS) * g
        if c["normed"]:
            out["normed"] = n.to(dt)
        return dict(out, values=_rounded(n, c["format"])) if c["format"] != "none" else out
    h, d = s["x"].float(), s["dnormed"].float()
    r = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    n = h * r
    dg = (d * n).sum(dim=0)
    d = d * g
    dh = r * (d - n * (d * n).mean(dim=1, keepdim=True))
    if c["residual"]:
        dh = dh + s["dsum"].float()
    out = {"dx": dh.to(dt), "dg": s["dg"].add_(dg) if c["accumulate"] else dg}
    return dict(out, dbranch=(dh * _factor(s)).to(dt)) if c["branch"] else out


# ------------------------------------------------------------------------------------------------- the library's kernels
_kept = {}   # what a program keeps: the context, one workspace


def _workspace(size):
    if _kept.get("size", -1) < size:
        _kept["ws"], _kept["size"] = torch.empty(size, dtype=torch.uint8, device=DEVICE), size
    return _kept["ws"]


def _own(s):
    from paper_2405_16256_amd import binding as hh
    c = s["case"]
    if "ctx" not in _kept:
        _kept["ctx"] = hh.hh_ctx_create(0)
    ctx, stream, rows, cols = _kept["ctx"], torch.cuda.current_stream().cuda_stream, c["rows"], c["cols"]
    dtype = hh.HH_BF16 if c["dtype"] == "bf16" else hh.HH_F32
    formats = {"none": hh.HH_MX_NONE, "e4m3": hh.HH_MX_E4M3, "e2m1": hh.HH_MX_E2M1}
    drop = hh.make_dropout(c["p"], s["seed"], s["offset"]) if c.get("p") else None
    if c["op"] == "dropout":
        hh.hh_dropout(ctx, drop, rows, cols, dtype, s["x"], cols, s["y"], cols, stream)
        return {"y": s["y"]}
    if c["op"] == "quantise":
        q = {k: hh.make_mx(*s[k]) for k in ("by_row", "by_column") if k in s}
        f, out = formats[c["format"]], {}
        hh.hh_mx_quantise(ctx, rows, cols, dtype, s["x"], cols, f, q.get("by_row"), q.get("by_column"), stream)
        if "by_row" in q:
            hh.hh_mx_values(ctx, rows, cols, f, q["by_row"], hh.HH_BF16, s["rows"], cols, stream)
            out["rows"] = s["rows"]
        if "by_column" in q:
            hh.hh_mx_values(ctx, cols, rows, f, q["by_column"], hh.HH_BF16, s["columns"], rows, stream)
            out["columns"] = s["columns"]
        return out
    if c["op"] == "product":
        cfg = hh.make_mx_product_cfg(rows, cols, c["inner"], formats[c["a"]], formats[c["b"]], dtype, cols)
        hh.hh_mx_product(ctx, cfg, hh.make_mx(*s["a"]), hh.make_mx(*s["b"]), s["out"], c["accumulate"],
                         _workspace(hh.hh_mx_product_sizes(cfg)), stream)
        return {"out": s["out"]}
    cfg = hh.make_add_norm_cfg(rows, cols, EPS, dtype, formats[c.get("format", "none")])
    if c["op"] == "norm":
        q = hh.make_mx(*s["packed"]) if "packed" in s else None
        hh.hh_add_norm_fwd(ctx, cfg, drop, s["x"], s["branch"], s["g"], s["sum"], s["normed"], q, stream)
        out = {k: s[k] for k in ("sum", "normed") if s[k] is not None}
        if q is None:
            return out
        hh.hh_mx_values(ctx, rows, cols, formats[c["format"]], q, hh.HH_BF16, s["values"], cols, stream)
        return dict(out, values=s["values"])
    hh.hh_add_norm_bwd(ctx, cfg, drop, s["x"], s["g"], s["dnormed"], s["dsum"], s["dx"], s["dbranch"], s["dg"], c["accumulate"],
                       _workspace(hh.hh_add_norm_sizes(cfg)), stream)
    out = {"dx": s["dx"], "dg": s["dg"]}
    return dict(out, dbranch=s["dbranch"]) if c["branch"] else out


def run(state):
    if own:
        return _own(state)
    return _plain(state)


# -------------------------------------------------------------------------------------------------- definition, 64 bits
def _kept_exactly(s):
    """0 or 1 over the share that is kept, on the host in unsigned 64 bits, then moved."""
    c = s["case"]
    t = round(c["p"] * 65536)
    if t == 0:
        return 1.0
    low, shift = np.uint64(0xFFFFFFFF), np.uint64(32)
    counter = np.zeros((4, c["rows"], (c["cols"] + 7) // 8), dtype=np.uint64)
    counter[0] += np.arange(counter.shape[2], dtype=np.uint64)[None, :]
    counter[1] += np.arange(c["rows"], dtype=np.uint64)[:, None]
    counter[2], counter[3] = s["offset"] % 2 ** 32, s["offset"] // 2 ** 32
    key = [s["seed"] % 2 ** 32, s["seed"] // 2 ** 32]
    for i in range(10):
        x, y = np.uint64((key[0] + i * 0x9E3779B9) % 2 ** 32), np.uint64((key[1] + i * 0xBB67AE85) % 2 ** 32)
        left, right = counter[0] * np.uint64(0xD2511F53), counter[2] * np.uint64(0xCD9E8D57)
        counter = np.stack(((right >> shift) ^ counter[1] ^ x, right & low, (left >> shift) ^ counter[3] ^ y, left & low))
    halves = np.ascontiguousarray(np.moveaxis(counter, 0, 2).astype("<u4")).view("<u2").reshape(c["rows"], -1)[:, :c["cols"]]
    return torch.from_numpy(halves >= t).to(DEVICE).double() / (1.0 - t / 65536)


def _nearest(x, format):
    """x in 64 bits on the numbers of the format, by a search among them, a block of 32 at a time."""
    f, top = FRACTION[format], TOP[format]
    numbers = [m * 2.0 ** (LEAST[format] - f) for m in range(1 << f)]
    numbers += [(1 + m / (1 << f)) * 2.0 ** e for e in range(LEAST[format], top + 1) for m in range(1 << f)]
    numbers = torch.tensor([v for v in numbers if v <= LARGEST[format]], dtype=torch.float64, device=DEVICE)
    between = (numbers[1:] + numbers[:-1]) / 2
    powers = torch.tensor([2.0 ** e for e in range(-126 + top, 128)], dtype=torch.float64, device=DEVICE)
    pieces = torch.split(x, BLOCK, dim=1)
    full = torch.nn.utils.rnn.pad_sequence([p.t() for p in pieces], batch_first=True) if x.shape[1] % BLOCK else torch.stack([p.t() for p in pieces])
    scale = torch.bucketize(full.abs().amax(dim=1), powers, right=True)   # blocks x rows: powers of two at or below the largest
    scale = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEVICE), scale - 127)[:, None, :]
    size = (full / scale).abs()
    down, up = torch.bucketize(size, between), torch.bucketize(size, between, right=True)
    found = numbers[torch.where(down % 2 == 0, down, up)] * torch.sign(full) * scale   # a tie: the even number
    return found.permute(2, 0, 1).reshape(x.shape[0], -1)[:, :x.shape[1]]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "dropout":
        return {"y": s["x"].double() * _kept_exactly(s)}
    if c["op"] == "quantise":
        x = s["x"].double()
        out = {} if c["by"] == "column" else {"rows": _nearest(x, c["format"])}
        return out if c["by"] == "row" else dict(out, columns=_nearest(x.t().contiguous(), c["format"]))
    if c["op"] == "product":
        tables = {"e2m1": torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64, device=DEVICE),
                  "e4m3": torch.arange(256, device=DEVICE).to(torch.uint8).view(torch.float8_e4m3fn).double()}
        sides = []
        for side in "ab":
            codes, scales = s[side]
            codes = codes.long()
            if c[side] == "e2m1":
                codes = torch.stack((codes % 16, codes // 16), dim=-1).flatten(1)
            power = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=DEVICE), scales.double() - 127)
            sides.append((tables[c[side]][codes] * power.repeat_interleave(BLOCK, dim=1))[:, :c["inner"]])
        y = torch.matmul(sides[0], sides[1].t())
        return {"out": y + s["out"].double() if c["accumulate"] else y}
    h, g = s["x"].double(), s["g"].double()
    if c["op"] == "norm":
        out = {}
        if c["branch"]:
            out["sum"] = h + s["branch"].double() * _kept_exactly(s)
            h = out["sum"].to(s["x"].dtype).double()   # the norm's operand is the sum as it is kept
        normed = h / torch.sqrt(torch.mean(h * h, dim=1, keepdim=True) + EPS) * g
        if c["normed"]:
            out["normed"] = normed
        return out if c["format"] == "none" else dict(out, values=_nearest(normed, c["format"]))
    d = s["dnormed"].double()
    root = torch.sqrt(torch.mean(h * h, dim=1, keepdim=True) + EPS)
    along = torch.sum(d * g * h, dim=1, keepdim=True) / h.shape[1]
    dx = d * g / root - h * along / root ** 3
    if c["residual"]:
        dx = dx + s["dsum"].double()
    dg = torch.sum(d * h / root, dim=0)
    out = {"dx": dx, "dg": dg + s["dg"].double() if c["accumulate"] else dg}
    return dict(out, dbranch=dx * _kept_exactly(s)) if c["branch"] else out
