"""Global gradient norm with clipping and the optimizer's update over lists of tensors, against plain numbers in 64 bits.

Tolerances, as relative Frobenius norms.  fp32 results: a few roundings of 2^-24 each, and the norm's one: 1e-6.  bf16
results: one rounding, at most 2^-8: 4e-3."""
import math

import pytest
import torch

from paper_2405_16256_amd import binding as hh

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP32, BF16 = 1e-6, 4e-3
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def ctx():
    c = hh.hh_ctx_create(0)
    yield c
    hh.hh_ctx_destroy(c)


def stream():
    return torch.cuda.current_stream().cuda_stream


def tensors(sizes, kind, offset, scale, gen):
    """Slices of one buffer, the first one `offset` elements behind its start, with elements that nothing may touch around each."""
    gap = 3
    flat = torch.randn(offset + sum(sizes) + gap * (len(sizes) + 1), device=DEV, generator=gen).mul_(scale).to(TYPES[kind])
    out, at = [], offset
    for n in sizes:
        out.append(flat[at:at + n])
        at += n + gap
    return flat, out


def off(got, ref):
    n = torch.linalg.vector_norm(ref)
    return float(torch.linalg.vector_norm(got.double() - ref) / (n if n > 0 else 1.0))


def outside(flat, parts):
    """The elements of the buffer that belong to no part."""
    mine = torch.zeros(flat.numel(), dtype=torch.bool, device=DEV)
    for p in parts:
        mine[p.storage_offset():p.storage_offset() + p.numel()] = True
    return flat[~mine]


# one element; no element; around the vectors, a workgroup's 256 threads and its chunk of 8192; more tensors than a launch takes (64, 48)
SIZES = [[1], [0], [], [0, 5, 0], [2, 3, 4, 5, 7, 8, 9], [255, 256, 257, 1023, 1025], [8191, 8192, 8193, 16385, 1], [300001, 17, 2000003],
         [1 + 37 * i % 411 for i in range(200)], [64] * 64, [64] * 65, [9] * 48 + [0] * 5 + [10000] * 49]


def clip(ctx, pairs, max_norm):
    result = torch.full((2,), 7.0, device=DEV)
    ws = torch.full((hh.HH_CLIP_WORKSPACE_BYTES,), 255, dtype=torch.uint8, device=DEV)
    hh.hh_grad_clip(ctx, hh.make_clip_tensors(pairs), max_norm, result, ws, stream())
    return result


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
@pytest.mark.parametrize("kind,offset", [("f32", 0), ("f32", 1), ("bf16", 0), ("bf16", 5)])
def test_norm_and_clipped_copies(ctx, sizes, kind, offset):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(len(sizes) + 3 * sum(sizes) + offset)
    _, g = tensors(sizes, kind, offset, 0.5, gen)
    ref = torch.sqrt(sum((t.double().square().sum() for t in g), torch.zeros((), dtype=torch.float64, device=DEV)))
    for max_norm in (0.25, 1e6):
        # copies in the same places of a buffer, in other places, in the gradients' own; norms alone for every other tensor
        for where in ("same", "shifted", "own", "some"):
            src = [t.clone() for t in g] if where == "own" else g
            flat, out = tensors(sizes, kind, offset + (where == "shifted"), 1.0, gen)
            around = outside(flat, out).clone()
            if where == "own":
                out = src
            pairs = [(a, None if where == "some" and i % 2 else b) for i, (a, b) in enumerate(zip(src, out))]
            left = [b.clone() for b in out]
            result = clip(ctx, pairs, max_norm)
            assert off(result[:1], ref[None]) <= FP32
            factor = min(1.0, max_norm / (float(ref) + 1e-6))
            assert abs(float(result[1]) - factor) <= FP32 * factor
            for (_, o), a, b, l in zip(pairs, g, out, left):
                if o is None:
                    assert torch.equal(b, l)
                elif b.numel():
                    assert off(b, a.double() * factor) <= (BF16 if kind == "bf16" else FP32)
            if where != "own":
                assert torch.equal(outside(flat, out), around)
    assert off(clip(ctx, [(t, None) for t in g], 1.0)[:1], ref[None]) <= FP32


def test_norm_of_mixed_types_and_of_extreme_values(ctx):
    a, b = torch.full((1000,), 1e30, device=DEV), torch.full((4001,), 1e30, dtype=torch.bfloat16, device=DEV)
    ref = math.sqrt(1000 * float(a[0]) ** 2 + 4001 * float(b[0]) ** 2)
    assert abs(float(clip(ctx, [(a, None), (b, None)], 1.0)[0]) - ref) <= FP32 * ref        # squares past the range of fp32
    a.fill_(1e-30)
    ref = math.sqrt(1000) * float(a[0])
    assert abs(float(clip(ctx, [(a, None)], 1.0)[0]) - ref) <= FP32 * ref                   # and below it
    for bad in (float("nan"), float("inf"), float("-inf")):
        a[17] = bad
        out = torch.zeros_like(a)
        result = clip(ctx, [(a, out)], 1.0)
        assert not torch.isfinite(result[0]) and torch.isnan(result[1]) and torch.isnan(out).all()


def test_norm_past_two_to_the_31_elements(ctx):
    n = 2 ** 31 + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    g[-1], g[2 ** 31 + 1], g[0] = 3.0, 4.0, 12.0
    assert float(clip(ctx, [(g, None)], 1.0)[0]) == 13.0
    clip(ctx, [(g, g)], 1.3)
    assert [round(float(g[i]), 2) for i in (0, 2 ** 31 + 1, n - 1)] == [1.2, 0.4, 0.3]


HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-6)


def update(p, m, v, g, factor, decay, step):
    g = g.double() * factor
    m = HYPER["beta1"] * m.double() + (1 - HYPER["beta1"]) * g
    v = HYPER["beta2"] * v.double() + (1 - HYPER["beta2"]) * g ** 2
    p = p.double()
    return p - HYPER["lr"] * (m / (1 - HYPER["beta1"] ** step) / (torch.sqrt(v / (1 - HYPER["beta2"] ** step)) + HYPER["eps"]) + decay * p), m, v


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%d_tensors_%d" % (len(s), sum(s)))
@pytest.mark.parametrize("param,grad,offset,apart", [("f32", "f32", 0, False), ("bf16", "f32", 0, False), ("bf16", "f32", 3, False), ("bf16", "bf16", 2, True),
                                                     ("f32", "bf16", 1, False), ("f32", "f32", 2, True)])
def test_update(ctx, sizes, param, grad, offset, apart):
    """apart: gradients lie another distance from 16 bytes than the rest, so that no vectors fit."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(len(sizes) + 3 * sum(sizes) + offset)
    flats, parts = zip(*[tensors(sizes, k, offset + (apart and i == 3), s, gen) for i, (k, s) in enumerate((("f32", 0.5), ("f32", 0.1), ("f32", 0.3), (grad, 0.2)))])
    p, m, v, g = parts
    for t in v:
        t.square_()
    copies, low = tensors(sizes, param, offset, 1.0, gen)
    around = [outside(f, x).clone() for f, x in zip(flats + (copies,), parts + (low,))]
    factor = torch.full((1,), 0.5, device=DEV)
    for step, f in ((1, None), (7, factor)):
        decay = [0.1 if i % 3 else 0.0 for i in range(len(sizes))]
        ref = [update(*t, 1.0 if f is None else 0.5, d, step) for t, d in zip(zip(p, m, v, g), decay)]
        rows = [(lo, a, b, c, d, w) if param == "bf16" else (a, None, b, c, d, w) for lo, a, b, c, d, w in zip(low, p, m, v, g, decay)]
        hh.hh_adamw_step(ctx, hh.make_adamw_cfg(step=step, **HYPER), hh.make_adamw_tensors(rows), f, stream())
        for got, want in zip(zip(p, m, v), ref):
            for a, b in zip(got, want):
                assert a.numel() == 0 or off(a, b) <= FP32
        if param == "bf16":
            assert all(torch.equal(lo, a.to(torch.bfloat16)) for lo, a in zip(low, p))
    assert all(torch.equal(outside(f, x), a) for f, x, a in zip(flats + (copies,), parts + (low,), around))


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_no_update_where_the_factor_is_not_finite(ctx, bad):
    t = [torch.rand(5000, device=DEV) for _ in range(4)]
    low = t[0].to(torch.bfloat16)
    was = [a.clone() for a in t + [low]]
    hh.hh_adamw_step(ctx, hh.make_adamw_cfg(step=1, **HYPER), hh.make_adamw_tensors([(low, *t, 0.1)]), torch.full((1,), bad, device=DEV), stream())
    assert all(torch.equal(a, b) for a, b in zip(t + [low], was))


def test_clipped_update_from_a_graph_and_on_another_stream(ctx):
    """Norm, factor and update one behind the other: replays give what the eager calls give."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    sizes = [5000, 17, 70001] * 40
    start = [tensors(sizes, "f32", 1, s, gen)[0] for s in (0.5, 0.1, 0.3, 0.2)]
    start[2].square_()
    work = [t.clone() for t in start]
    split = lambda t: torch.split(t[:sum(sizes)], sizes)  # noqa: E731
    result, ws = torch.empty(2, device=DEV), torch.empty(hh.HH_CLIP_WORKSPACE_BYTES, dtype=torch.uint8, device=DEV)
    clips = hh.make_clip_tensors([(g, None) for g in split(work[3])])
    rows = hh.make_adamw_tensors([(a, None, b, c, d, 0.1) for a, b, c, d in zip(*map(split, work))])

    def call():
        hh.hh_grad_clip(ctx, clips, 1.0, result, ws, stream())
        hh.hh_adamw_step(ctx, hh.make_adamw_cfg(step=3, **HYPER), rows, result[1:], stream())

    call()
    want = [t.clone() for t in work]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t, s in zip(work, start):
            t.copy_(s)
        call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(work, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t, s in zip(work, start):
            t.copy_(s)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(work, want))
