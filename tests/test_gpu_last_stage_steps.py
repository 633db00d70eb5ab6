"""Steps of a pipeline's last stage that do not go by the book: labels past the vocabulary, gradients that are not finite."""
import pytest
import torch

from paper_2405_16256_amd import glue as L
from paper_2405_16256_amd import inputs as I
from paper_2405_16256_amd import last_stage as S

pytestmark = pytest.mark.gpu
SHAPE, VOCAB, SEED = I.LayerShape(256, 4, 64, 704, 60, 2), 301, 5


def stage_and_batch(bf16, **kw):
    head = I.normal(SEED, S.TID_HEAD, (VOCAB, SHAPE.hidden), scale=0.02)
    stage = S.LastStage(SHAPE, [I.layer_weights(SEED, l, SHAPE, bf16) for l in range(2)], head, bf16, **kw)
    x, labels = S.batch(SEED, SHAPE, VOCAB, 2, bf16)
    x = [L.to_dev(t, bf16) for t in x]
    return stage, x, [torch.from_numpy(t).to(L.DEV) for t in labels], [torch.empty(SHAPE.tokens, device=L.DEV) for _ in x], [torch.empty_like(t) for t in x]


@pytest.mark.parametrize("bf16", [False, True])
def test_labels_past_the_vocabulary_do_not_count(bf16):
    """The gradients are those of the mean over the other tokens, bit for bit what negative labels give."""
    stage, x, labels, losses, dx = stage_and_batch(bf16)
    found = []
    for label in (-100, VOCAB, 2 ** 40):
        for t in labels:
            t[5:25] = label
        stage.gradients(x, labels, losses, dx)
        found.append([g.clone() for _, g, _ in stage.params] + [t.clone() for t in dx])
        for t in losses:
            assert (t[5:25] == 0).all() if label < 0 else torch.isnan(t[5:25]).all()
    for other in found[1:]:
        assert all(torch.equal(a, b) for a, b in zip(found[0], other))
    stage.close()


def test_gradients_do_not_wait_for_the_device():
    stage, x, labels, losses, dx = stage_and_batch(True)
    stage.gradients(x, labels, losses, dx)
    torch.cuda.synchronize()
    was = torch.cuda.get_sync_debug_mode()
    torch.cuda.set_sync_debug_mode("error")
    try:
        stage.gradients(x, labels, losses, dx)
    finally:
        torch.cuda.set_sync_debug_mode(was)
    stage.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_step_that_is_left_out_does_not_count(bad):
    """A gradient that is not finite: nothing changes, and the steps behind it are those of a run without it, bit for bit."""
    stage, x, labels, losses, dx = stage_and_batch(True)
    other = stage_and_batch(True)[0]
    for s in (stage, other):
        for step in range(4):
            s.gradients(x, labels, losses, dx)
            if step in (1, 2):
                if s is other:
                    continue
                s.params[3][1].view(-1)[7] = bad
                state = [t.clone() for t in (*s.masters, *(p for p, _, _ in s.params), *(m for pair in s.moments for m in pair))]
                s.update()
                assert all(torch.equal(a, b) for a, b in zip(state, (*s.masters, *(p for p, _, _ in s.params), *(m for pair in s.moments for m in pair))))
                continue
            s.update()
        assert s.step_no == 2
    for a, b in zip(stage.masters, other.masters):
        assert torch.equal(a, b)
    for a, b in zip(stage.moments, other.moments):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(torch.equal(a[0], b[0]) for a, b in zip(stage.params, other.params))
    stage.close()
    other.close()
