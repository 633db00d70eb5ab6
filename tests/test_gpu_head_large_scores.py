"""Output projection with softmax cross entropy where scores are large, tied or certain, and where labels lie past the vocabulary, on
rows of every length: those that one workgroup holds whole, longer ones, and shares of a vocabulary.

Every score here is a multiple of 1/4 below 2^14 and every product exact, so the device's scores are the exact ones and what is off is
the softmax's own arithmetic.  A token's row of x is its offset in column 0, the same for all words, and a one in a column of its
own: that column of dW is the token's d.

Tolerances.  FP32 and BF16 as relative errors, for sums of fp32 numbers, d as two bf16 numbers (at most 2^-16 = 1.5e-5) and dx in bf16.
CANCEL: p of the label, 1 in the worst case, has a rounding of 2^-24 from each of the exponential, the sum, its reciprocal and the
product, and d = p - 1 keeps them; log of the sum likewise: 2^-22."""
import pytest
import torch

from paper_2405_16256_amd import binding as hh

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, hh.HH_BF16), "f32": (torch.float32, hh.HH_F32)}
FP32, BF16, CANCEL = 2e-5, 5e-3, 2.0 ** -22
OFFSETS = (0.0, 100.0, 1000.0, -1000.0, 12736.0, -12736.0)
HIDDEN, TOKENS = 64, 60
# a row is in one workgroup up to 16384 words (fp32 32768)
KINDS = [("bf16", 1001), ("bf16", 20011), ("f32", 1001), ("f32", 33001)]


@pytest.fixture(scope="module")
def ctx():
    c = hh.hh_ctx_create(0)
    yield c
    hh.hh_ctx_destroy(c)


def stream():
    return torch.cuda.current_stream().cuda_stream


def case(kind, vocab):
    """x, w, labels: each offset with tokens whose scores are spread, tied between two words, or certain."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(vocab)
    w = torch.randint(-32, 33, (vocab, HIDDEN), device=DEV, generator=gen) / 4.0
    w[:, 0] = 1.0
    labels = torch.randint(0, vocab, (TOKENS,), device=DEV, generator=gen)
    x = torch.zeros(TOKENS, HIDDEN, device=DEV)
    for t in range(TOKENS):
        x[t, 0], x[t, 1 + t] = OFFSETS[t % len(OFFSETS)], 1.0
        shape = t // len(OFFSETS) % 3
        if shape == 1:      # two words share the probability
            w[labels[t], 1 + t] = w[(int(labels[t]) + vocab // 2) % vocab, 1 + t] = 30.0
        elif shape == 2:    # certain
            w[labels[t], 1 + t] = 30.0
    dt = TYPES[kind][0]
    assert torch.equal(x.to(dt).float(), x) and torch.equal(w.to(dt).float(), w)
    return x.to(dt), w.to(dt), labels


def definition(x, w, labels):
    """(loss, d, p, lse) in 64 bits, with the label's d as the sum of the others."""
    z = x.double() @ w.double().t()
    rows = torch.arange(len(x), device=DEV)
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    p = e / e.sum(1, keepdim=True)
    d = p.clone()
    d[rows, labels] = 0.0
    rest = d.sum(1)
    d[rows, labels] = -rest
    loss = torch.where(rest < 0.5, -torch.log1p(-rest), -torch.log(p[rows, labels]))
    return loss, d, p, top[:, 0] + torch.log(e.sum(1))


def check_gradients(kind, x, w, d, dx, dw, off):
    """off[t]: what d of token t may be off by (2-norm)."""
    x, w = x.double(), w.double()
    assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
    err = torch.linalg.vector_norm(dw.double() - d.t() @ x, dim=0)
    assert (err <= x.abs().t() @ off).all(), (err / (x.abs().t() @ off)).max()
    size = torch.linalg.vector_norm(w, dim=1)
    err = torch.linalg.vector_norm(dx.double() - d @ w, dim=1)
    most = (BF16 if kind == "bf16" else FP32) * (d.abs() @ size) + off * size.max()
    assert (err <= most).all(), (err / most).max()


def filled(n):
    return torch.full((n,), 255, dtype=torch.uint8, device=DEV)   # NaNs


@pytest.mark.parametrize("kind,vocab", KINDS)
def test_large_tied_and_certain_scores(ctx, kind, vocab):
    x, w, labels = case(kind, vocab)
    ref, d, _, _ = definition(x, w, labels)
    cfg = hh.make_head_cfg(HIDDEN, vocab, TOKENS, TYPES[kind][1])
    sizes = hh.hh_head_sizes(cfg)
    alone, loss = torch.full((TOKENS,), 7.0, device=DEV), torch.full((TOKENS,), 7.0, device=DEV)
    dx, dw = torch.full_like(x, 7.0), torch.full((vocab, HIDDEN), 7.0, device=DEV)
    hh.hh_head_loss(ctx, cfg, x, w, labels, alone, filled(sizes[0]), stream())
    hh.hh_head_step(ctx, cfg, x, w, labels, None, 1.0, loss, dx, dw, 0, filled(sizes[1]), stream())
    for got in (alone, loss):
        err = (got.double() - ref).abs()
        assert (err <= FP32 * ref + CANCEL).all(), (err / (FP32 * ref + CANCEL)).max()
    check_gradients(kind, x, w, d, dx, dw, FP32 * torch.linalg.vector_norm(d, dim=1) + CANCEL)


@pytest.mark.parametrize("kind,vocab", KINDS)
def test_labels_past_the_vocabulary(ctx, kind, vocab):
    """Such a loss is NaN, and the token adds no gradient; the others are as without it."""
    x, w, labels = case(kind, vocab)
    cfg = hh.make_head_cfg(HIDDEN, vocab, TOKENS, TYPES[kind][1])
    sizes = hh.hh_head_sizes(cfg)
    bad = {7: vocab, 8: vocab + 1, 20: 2 ** 31, 21: 2 ** 40 + 5, 33: 2 ** 63 - 1}
    none = {40: -1, 41: -100, 42: -2 ** 40, 43: -2 ** 63}
    counts = torch.ones(TOKENS, dtype=torch.bool, device=DEV)
    named = labels.clone()
    for t, v in {**bad, **none}.items():
        named[t], counts[t] = v, False
    ref, d, _, _ = definition(x, w, labels)
    d[~counts] = 0.0
    alone, loss = torch.full((TOKENS,), 7.0, device=DEV), torch.full((TOKENS,), 7.0, device=DEV)
    dx, dw = torch.full_like(x, 7.0), torch.full((vocab, HIDDEN), 7.0, device=DEV)
    hh.hh_head_loss(ctx, cfg, x, w, named, alone, filled(sizes[0]), stream())
    hh.hh_head_step(ctx, cfg, x, w, named, None, 1.0, loss, dx, dw, 0, filled(sizes[1]), stream())
    for got in (alone, loss):
        assert torch.isnan(got[list(bad)]).all() and (got[list(none)] == 0).all()
        assert ((got.double() - ref).abs() <= FP32 * ref + CANCEL)[counts].all()
    assert (dx[~counts] == 0).all()
    off = FP32 * torch.linalg.vector_norm(d, dim=1) + CANCEL * counts
    check_gradients(kind, x, w, d, dx, dw, off)


@pytest.mark.parametrize("kind,vocab", KINDS)
def test_shares_are_off_by_the_rounding_of_their_lse(ctx, kind, vocab):
    """What the shares tell each other is one fp32 number a token: rounded in each share and again for all of them, it moves the loss by
    2^-23 |lse| at most and p by as much of itself."""
    x, w, labels = case(kind, vocab)
    ref, d, p, lse64 = definition(x, w, labels)
    cuts, total, picked = (0, vocab // 3, vocab), None, 0.0
    cfgs = [hh.make_head_cfg(HIDDEN, b - a, TOKENS, TYPES[kind][1]) for a, b in zip(cuts, cuts[1:])]
    for cfg, a, b in zip(cfgs, cuts, cuts[1:]):
        s, q = (torch.full((TOKENS,), 7.0, device=DEV) for _ in range(2))
        hh.hh_head_share_fwd(ctx, cfg, x, w[a:b].clone(), labels, a, s, q, filled(hh.hh_head_sizes(cfg)[0]), stream())
        total = s.double() if total is None else torch.logaddexp(total, s.double())
        picked = picked + q.double()
    lse = total.float()
    moved = 2.0 ** -23 * lse64.abs()
    err = (lse.double() - picked - ref).abs()
    assert (err <= FP32 * ref + CANCEL + moved).all()
    dw = torch.full((vocab, HIDDEN), 7.0, device=DEV)
    for cfg, a, b in zip(cfgs, cuts, cuts[1:]):
        dx, part = torch.full_like(x, 7.0), torch.full((b - a, HIDDEN), 7.0, device=DEV)
        hh.hh_head_share_bwd(ctx, cfg, x, w[a:b].clone(), labels, a, lse, None, 1.0, dx, part, 0, filled(hh.hh_head_sizes(cfg)[1]), stream())
        dw[a:b] = part
        off = FP32 * torch.linalg.vector_norm(d, dim=1) + CANCEL + moved * torch.linalg.vector_norm(p, dim=1)
        check_gradients(kind, x, w[a:b], d[:, a:b], dx, part, off)
