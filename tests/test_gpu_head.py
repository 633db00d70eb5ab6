"""Output projection with softmax cross entropy (hh_head_loss, hh_head_step) against the definition in 64 bits.

Tolerances, as relative Frobenius norms.  fp32 quantities (losses, every fp32 result): sums of up to 10^5 products of fp32
numbers, each rounded at 2^-24 and errors adding up as the root of their number at worst: 2e-5.  dx in bf16: d and the result
rounded once each, 1.7e-3 in the mean square (at most 2^-8), together below 5e-3.  dW in bf16: d as two bf16 numbers, at most 2^-16 =
1.5e-5 and 2.8e-6 in the mean square, and fp32 sums: 2e-5."""
import numpy as np
import pytest
import torch

from paper_2405_16256_amd import binding as hh

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FP32, BF16 = 2e-5, 5e-3


@pytest.fixture(scope="module")
def ctx():
    c = hh.hh_ctx_create(0)
    yield c
    hh.hh_ctx_destroy(c)


def stream():
    return torch.cuda.current_stream().cuda_stream


def inputs(kind, hidden, vocab, tokens, ignored=0.2, seed=0):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000 * seed + hidden + 7 * vocab + 31 * tokens)
    rand = lambda *s: torch.randn(*s, device=DEV, generator=gen)  # noqa: E731
    w = (rand(vocab, hidden) * 1.5 / hidden ** 0.5).to(TYPES[kind])
    labels = torch.randint(0, vocab, (tokens,), device=DEV, generator=gen)
    x = (rand(tokens, hidden) + w[labels].float()).to(TYPES[kind])
    labels[torch.rand(tokens, device=DEV, generator=gen) < ignored] = -100
    return x, w, labels


def definition(x, w, labels, g):
    """(loss, dx, dw) in 64 bits; g: upstream gradient of each loss."""
    x, w, g = x.double(), w.double(), g.double()
    counts = ((labels >= 0) & (labels < w.shape[0])).nonzero()[:, 0]
    loss, dx = torch.zeros(len(x), dtype=torch.float64, device=DEV), torch.zeros_like(x)
    z = x[counts] @ w.t()
    lse = torch.logsumexp(z, 1)
    at = (torch.arange(len(counts), device=DEV), labels[counts])
    loss[counts] = lse - z[at]
    d = torch.exp(z - lse[:, None])
    d[at] -= 1
    d *= g[counts][:, None]
    dx[counts] = d @ w
    return loss, dx, d.t() @ x[counts]


def step(ctx, kind, x, w, labels, dloss=None, scale=1.0, dw=None, dx=None):
    (tokens, hidden), vocab = x.shape, w.shape[0]
    cfg = hh.make_head_cfg(hidden, vocab, tokens, hh.HH_BF16 if kind == "bf16" else hh.HH_F32)
    loss = torch.full((tokens,), 7.0, device=DEV)
    dx = torch.full_like(x, 7.0) if dx is None else dx
    acc = dw is not None
    dw = torch.full((vocab, hidden), 7.0, device=DEV) if dw is None else dw
    ws = torch.full((hh.hh_head_sizes(cfg)[1],), 255, dtype=torch.uint8, device=DEV)   # NaNs
    hh.hh_head_step(ctx, cfg, x, w, labels, dloss, scale, loss, dx, dw, acc, ws, stream())
    return loss, dx, dw


def loss_of(ctx, kind, x, w, labels):
    (tokens, hidden), vocab = x.shape, w.shape[0]
    cfg = hh.make_head_cfg(hidden, vocab, tokens, hh.HH_BF16 if kind == "bf16" else hh.HH_F32)
    loss = torch.full((tokens,), 7.0, device=DEV)
    ws = torch.full((hh.hh_head_sizes(cfg)[0],), 255, dtype=torch.uint8, device=DEV)
    hh.hh_head_loss(ctx, cfg, x, w, labels, loss, ws, stream())
    return loss


def off(got, ref):
    n = torch.linalg.vector_norm(ref)
    return float(torch.linalg.vector_norm(got.double() - ref) / (n if n > 0 else 1.0))


def check(kind, got, ref):
    for name, a, b in zip(("loss", "dx", "dw"), got, ref):
        assert torch.isfinite(a).all(), name
        assert off(a, b) <= (BF16 if name == "dx" and kind == "bf16" else FP32), (name, off(a, b))


# one token and one word; around the slots of 64 columns, the tiles of 64, 128 and 256 rows and columns, k of one and several stages;
# each tile that the product of the scores is launched with; vocabularies past 65536
SHAPES = [("bf16", 64, 1, 1), ("bf16", 64, 2, 1), ("bf16", 64, 63, 5), ("bf16", 128, 65, 64), ("bf16", 192, 127, 65), ("bf16", 256, 1000, 129),
          ("bf16", 320, 1001, 257), ("bf16", 512, 5003, 300), ("bf16", 1024, 20011, 333), ("bf16", 2048, 8191, 1100), ("bf16", 128, 100003, 70),
          ("bf16", 4096, 32000, 513), ("bf16", 64, 257, 4099),
          ("f32", 8, 1, 1), ("f32", 8, 3, 2), ("f32", 40, 63, 5), ("f32", 64, 65, 33), ("f32", 256, 1000, 128), ("f32", 136, 1025, 65),
          ("f32", 1024, 4099, 200), ("f32", 16, 70001, 19), ("f32", 360, 19739, 11), ("f32", 104, 2501, 300), ("f32", 72, 131, 2051)]


@pytest.mark.parametrize("kind,hidden,vocab,tokens", SHAPES)
def test_loss_and_gradients(ctx, kind, hidden, vocab, tokens):
    x, w, labels = inputs(kind, hidden, vocab, tokens, 0.0 if tokens < 4 else 0.2)
    scale = 1.0 / tokens
    ref = definition(x, w, labels, torch.full((tokens,), scale, device=DEV))
    check(kind, step(ctx, kind, x, w, labels, scale=scale), ref)
    assert off(loss_of(ctx, kind, x, w, labels), ref[0]) <= FP32


@pytest.mark.parametrize("kind,hidden,vocab,tokens", [("bf16", 256, 1001, 100), ("f32", 72, 503, 100), ("bf16", 1024, 9001, 700)])
def test_upstream_gradients_and_sums(ctx, kind, hidden, vocab, tokens):
    """A gradient for each token's loss, dW added to what is there, dx in x's own place."""
    x, w, labels = inputs(kind, hidden, vocab, tokens)
    dloss = torch.randn(tokens, device=DEV)
    dloss[labels < 0] = float("nan")        # what does not count is not looked at
    ref = definition(x, w, labels, 0.25 * torch.nan_to_num(dloss))
    before = torch.randn(vocab, hidden, device=DEV) * 0.01
    same = x.clone()
    loss, dx, dw = step(ctx, kind, same, w, labels, dloss, 0.25, before.clone(), dx=same)
    check(kind, (loss, dx, dw), (ref[0], ref[1], ref[2] + before.double()))


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_tokens_that_do_not_count(ctx, kind):
    """Negative labels: loss and gradient are zero, whatever the row holds; a label past the vocabulary: NaN, and no gradient."""
    hidden, vocab, tokens = 128, 300, 70
    x, w, labels = inputs(kind, hidden, vocab, tokens, 0.0)
    labels[3], labels[9], labels[10], labels[11], labels[64] = -1, -100, -2 ** 40, -5, -3
    x[9], x[10], x[64, 5] = float("nan"), float("inf"), float("-inf")
    clean = x.clone()
    clean[labels < 0] = 0
    ref = definition(clean, w, labels, torch.ones(tokens, device=DEV))
    got = step(ctx, kind, x, w, labels)
    check(kind, got, ref)
    assert (got[0][labels < 0] == 0).all() and (got[1][labels < 0] == 0).all()
    assert (loss_of(ctx, kind, x, w, labels)[labels < 0] == 0).all()
    for bad in (vocab, vocab + 1, 2 ** 31, 2 ** 40 + 5):
        labels[20] = bad
        ref = definition(clean, w, labels, torch.ones(tokens, device=DEV))
        loss, dx, dw = step(ctx, kind, x, w, labels)
        assert torch.isnan(loss[20]) and int(torch.isnan(loss).sum()) == 1
        loss[20] = 0
        check(kind, (loss, dx, dw), ref)
    labels[:] = -100                         # no token counts
    loss, dx, dw = step(ctx, kind, x, w, labels)
    assert (loss == 0).all() and (dx == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_extreme_scores(ctx, kind):
    """Scores of thousands, a certain answer, equal scores, scores of -inf in some columns, infinite or NaN hidden states."""
    hidden, vocab, tokens = 64, 200, 8
    x = torch.zeros(tokens, hidden, dtype=TYPES[kind], device=DEV)
    w = torch.zeros(vocab, hidden, dtype=TYPES[kind], device=DEV)
    labels = torch.arange(tokens, device=DEV)
    w[:, 0] = torch.arange(vocab, device=DEV).to(TYPES[kind])
    x[1, 0], x[2, 0], x[3, 0] = 64.0, -64.0, 2.0 ** 100
    w[5, 1], x[5, 1] = 50.0, 1.0             # certain
    ref = definition(x, w, labels, torch.ones(tokens, device=DEV))
    got = step(ctx, kind, x, w, labels)
    check(kind, got, ref)
    assert abs(float(got[0][0]) - float(np.log(vocab))) < 1e-5
    # scores that overflow to -inf are columns of no weight; +inf or NaN makes the loss NaN, of this token alone
    big = 3e38
    x2, w2 = x.clone(), w.clone()
    w2[:, 2], w2[7, 2] = -big, 0.0
    x2[4, 2] = big
    labels[4] = 7
    x2[6, 0] = float("nan")
    loss = loss_of(ctx, kind, x2, w2, labels)
    assert abs(float(loss[4])) < 1e-6 and torch.isnan(loss[6])
    keep = torch.tensor([0, 1, 2, 3, 5, 7], device=DEV)
    assert off(loss[keep], definition(x2[keep], w2, labels[keep], torch.ones(6, device=DEV))[0]) <= FP32


def test_blocks_of_tokens(ctx):
    """More tokens than a block holds (32768): dW is the sum over the blocks."""
    x, w, labels = inputs("bf16", 64, 130, 70001, 0.1)
    ref = definition(x, w, labels, torch.full((70001,), 1e-3, device=DEV))
    check("bf16", step(ctx, "bf16", x, w, labels, scale=1e-3), ref)
    x, w, labels = inputs("f32", 8, 60, 40000, 0.1)
    ref = definition(x, w, labels, torch.full((40000,), 1e-3, device=DEV))
    check("f32", step(ctx, "f32", x, w, labels, scale=1e-3), ref)
    assert off(loss_of(ctx, "f32", x, w, labels), ref[0]) <= FP32


def test_pieces_of_the_vocabulary(ctx):
    """A gradient of more than 2^31 bytes is written in pieces of the vocabulary, the scores of a block in pieces of the tokens."""
    hidden, vocab, tokens = 4096, 132000, 700
    x, w, labels = inputs("bf16", hidden, vocab, tokens, 0.1)
    ref = definition(x, w, labels, torch.full((tokens,), 1.0 / tokens, device=DEV))
    check("bf16", step(ctx, "bf16", x, w, labels, scale=1.0 / tokens), ref)


# shares of one word, of no whole slot, that begin and end inside slots and tiles; past 32768 words; none but one share
@pytest.mark.parametrize("kind,hidden,tokens,cuts", [("bf16", 64, 70, [0, 1, 64, 130]), ("bf16", 512, 300, [0, 2500, 5003]), ("bf16", 256, 129, [0, 300, 40001]),
                                                     ("bf16", 1024, 700, [0, 12500, 25000, 37500, 50001]), ("f32", 40, 33, [0, 7, 8, 1200]),
                                                     ("f32", 256, 128, [0, 1000]), ("f32", 64, 50, [0, 33000, 40001])])
def test_shares_of_the_vocabulary(ctx, kind, hidden, tokens, cuts):
    """Each share by itself; the sums over the shares are those of the whole vocabulary.  dx: a share's partial sum is rounded once, so
    the total is off by as much of the partial sums as each of them may be."""
    vocab = cuts[-1]
    x, w, labels = inputs(kind, hidden, vocab, tokens)
    labels[::7] = torch.tensor([cuts[1 % (len(cuts) - 1)], vocab - 1, 0], device=DEV).repeat(tokens)[:len(labels[::7])]   # the shares' first and last words
    x[labels < 0] = float("nan")
    dloss = torch.rand(tokens, device=DEV)
    loss, dx, dw = definition(torch.nan_to_num(x), w, labels, 0.5 * dloss)
    found, lse = [], torch.full((tokens,), float("-inf"), device=DEV, dtype=torch.float64)
    for a, b in zip(cuts, cuts[1:]):
        cfg = hh.make_head_cfg(hidden, b - a, tokens, hh.HH_BF16 if kind == "bf16" else hh.HH_F32)
        sizes = hh.hh_head_sizes(cfg)
        s, picked = (torch.full((tokens,), 7.0, device=DEV) for _ in range(2))
        share = w[a:b].clone()
        hh.hh_head_share_fwd(ctx, cfg, x, share, labels, a, s, picked, torch.full((sizes[0],), 255, dtype=torch.uint8, device=DEV), stream())
        here = (labels >= a) & (labels < b)
        assert (picked[~here] == 0).all()
        lse = torch.where(labels >= 0, torch.logaddexp(lse, s.double()), torch.zeros_like(lse))
        found.append((cfg, sizes, share, a, b, picked))
    total = torch.where(labels >= 0, lse - sum(f[5].double() for f in found), torch.zeros_like(lse))
    assert off(total, loss) <= FP32
    lse = lse.float()
    lse[labels < 0] = float("nan")           # what does not count is not looked at
    got, partial = torch.zeros(tokens, hidden, device=DEV, dtype=torch.float64), 0.0
    for cfg, sizes, share, a, b, _ in found:
        dxs, before = torch.full_like(x, 7.0), torch.randn(b - a, hidden, device=DEV) * 0.01
        dws = before.clone()
        hh.hh_head_share_bwd(ctx, cfg, x, share, labels, a, lse, dloss, 0.5, dxs, dws, True, torch.full((sizes[1],), 255, dtype=torch.uint8, device=DEV), stream())
        assert off(dws, dw[a:b] + before.double()) <= FP32
        assert (dxs[labels < 0] == 0).all()
        got += dxs.double()
        partial += float(torch.linalg.vector_norm(dxs.double()))
    assert float(torch.linalg.vector_norm(got - dx)) <= (BF16 if kind == "bf16" else FP32) * partial


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_differences(ctx, kind):
    """Both gradients against differences of the loss itself, taken in 64 bits along random directions."""
    x, w, labels = inputs(kind, 64, 101, 9, 0.2)
    g = torch.rand(9, device=DEV)
    _, dx, dw = step(ctx, kind, x, w, labels, g)
    total = lambda x, w: float((definition(x, w, labels, g)[0] * g.double()).sum())  # noqa: E731
    for seed in range(3):
        gen = torch.Generator(device=DEV)
        gen.manual_seed(seed)
        ux, uw = (torch.randn(t.shape, device=DEV, dtype=torch.float64, generator=gen) for t in (x, w))
        e = 1e-5
        along = (total(x.double() + e * ux, w.double()) - total(x.double() - e * ux, w.double())) / (2 * e)
        assert abs(float((dx.double() * ux).sum()) - along) <= (BF16 if kind == "bf16" else FP32) * float(torch.linalg.vector_norm(dx.double()) * torch.linalg.vector_norm(ux))
        along = (total(x.double(), w.double() + e * uw) - total(x.double(), w.double() - e * uw)) / (2 * e)
        assert abs(float((dw.double() * uw).sum()) - along) <= FP32 * float(torch.linalg.vector_norm(dw.double()) * torch.linalg.vector_norm(uw))


@pytest.mark.parametrize("kind,hidden,vocab,tokens", [("bf16", 512, 5003, 300), ("bf16", 2048, 32000, 1100), ("f32", 256, 1000, 128)])
def test_same_bits_again_on_another_stream_and_from_a_graph(ctx, kind, hidden, vocab, tokens):
    x, w, labels = inputs(kind, hidden, vocab, tokens)
    want = [t.clone() for t in step(ctx, kind, x, w, labels)]
    cfg = hh.make_head_cfg(hidden, vocab, tokens, hh.HH_BF16 if kind == "bf16" else hh.HH_F32)
    ws = torch.empty(hh.hh_head_sizes(cfg)[1], dtype=torch.uint8, device=DEV)
    out = [torch.empty_like(t) for t in want]

    def call():
        hh.hh_head_step(ctx, cfg, x, w, labels, None, 1.0, out[0], out[1], out[2], False, ws, stream())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in out:
            t.zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        step(ctx, kind, x, w, labels)        # eager work in between


def test_work_is_traced(ctx):
    x, w, labels = inputs("bf16", 256, 1001, 100)
    hh.hh_trace_begin(ctx, 64)
    step(ctx, "bf16", x, w, labels)
    got = hh.hh_trace_end(ctx)
    for kind in ("gemm_nt", "gemm_nn", "gemm_tn"):
        assert got[kind][0] == 1 and got[kind][2] == 2.0 * 100 * 256 * 1001
    assert got["elementwise"][0] == 1
