"""Lists of as many tensors as a launch of clipping (112) or of the update (56) takes, one fewer, one more and several times as many, with
and without empty tensors behind them, against plain numbers in 64 bits.

Tolerances, as relative Frobenius norms: fp32 a few roundings of 2^-24 each, 1e-6; bf16 one rounding, at most 2^-8: 4e-3."""
import pytest
import torch

from paper_2405_16256_amd import binding as hh

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FP32, BF16 = 1e-6, 4e-3
COUNTS = [55, 56, 57, 111, 112, 113, 168, 224, 225]


@pytest.fixture(scope="module")
def ctx():
    c = hh.hh_ctx_create(0)
    yield c
    hh.hh_ctx_destroy(c)


def stream():
    return torch.cuda.current_stream().cuda_stream


def off(got, ref):
    n = torch.linalg.vector_norm(ref)
    return float(torch.linalg.vector_norm(got.double() - ref) / (n if n > 0 else 1.0))


def sizes(n, empty):
    """n tensors of 1 to 9000 elements; empty ones in front of, between and behind them."""
    out = [1 + 977 * i * i % 9000 for i in range(n)]
    return out if not empty else [0] + out[:n // 2] + [0, 0] + out[n // 2:] + [0] * 3


@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("n", COUNTS)
def test_clipping(ctx, n, empty):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    g = [torch.randn(k, device=DEV, generator=gen).to(torch.bfloat16 if i % 3 == 1 else torch.float32) for i, k in enumerate(sizes(n, empty))]
    ref = torch.sqrt(sum(t.double().square().sum() for t in g))
    ws = torch.full((hh.HH_CLIP_WORKSPACE_BYTES,), 255, dtype=torch.uint8, device=DEV)
    for copies in (0, 1, 5):     # none, each, some
        out = [torch.full_like(t, 7.0) if copies and i % copies == 0 else None for i, t in enumerate(g)]
        result = torch.full((2,), 7.0, device=DEV)
        hh.hh_grad_clip(ctx, hh.make_clip_tensors(list(zip(g, out))), 0.5, result, ws, stream())
        factor = 0.5 / (float(ref) + 1e-6)
        assert off(result[:1], ref[None]) <= FP32 and abs(float(result[1]) - factor) <= FP32 * factor
        for a, b in zip(g, out):
            if b is not None and b.numel():
                assert off(b, a.double() * factor) <= (BF16 if a.dtype == torch.bfloat16 else FP32)


@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("n", COUNTS)
def test_update(ctx, n, empty):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    lr, b1, b2, eps, step = 1e-2, 0.9, 0.95, 1e-6, 3
    rows, refs = [], []
    for i, k in enumerate(sizes(n, empty)):
        p, m, v, g = (torch.randn(k, device=DEV, generator=gen) for _ in range(4))
        v.square_()
        g = g.to(torch.bfloat16) if i % 4 == 2 else g
        decay = 0.1 * (i % 2)
        low = p.to(torch.bfloat16) if i % 3 == 1 else None
        rows.append((p, None, m, v, g, decay) if low is None else (low, p, m, v, g, decay))
        d = g.double()
        rm, rv = b1 * m.double() + (1 - b1) * d, b2 * v.double() + (1 - b2) * d ** 2
        rp = p.double() - lr * (rm / (1 - b1 ** step) / (torch.sqrt(rv / (1 - b2 ** step)) + eps) + decay * p.double())
        refs.append((p, m, v, low, rp, rm, rv))
    hh.hh_adamw_step(ctx, hh.make_adamw_cfg(lr, b1, b2, eps, step), hh.make_adamw_tensors(rows), None, stream())
    for p, m, v, low, rp, rm, rv in refs:
        if p.numel():
            assert off(p, rp) <= FP32 and off(m, rm) <= FP32 and off(v, rv) <= FP32
            assert low is None or torch.equal(low, p.to(torch.bfloat16))
