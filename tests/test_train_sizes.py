"""hh_head_sizes: the bounds of the workspaces that the header states, over sizes up to the largest.  Runs without a GPU."""
import pytest

from paper_2405_16256_amd import binding as hh

GIB, MIB = 1 << 30, 1 << 20
HIDDEN = (64, 1024, 4096, 8192, 16384, 24576, 32768)
VOCAB = (1, 64, 1000, 16320, 16384, 24576, 32000, 32704, 32769, 65536, 100003, 262144)
TOKENS = (1, 255, 4096, 16383, 16384, 20000, 32767, 32768, 65000, 200000, 1 << 20, 1 << 24)


@pytest.mark.parametrize("dtype,most_loss,most_step", [(hh.HH_BF16, 65 * MIB, int(4.6 * GIB)), (hh.HH_F32, int(2.01 * GIB), int(4.1 * GIB))])
def test_workspaces_are_bounded(dtype, most_loss, most_step):
    seen = 0
    for hidden in HIDDEN:
        for vocab in VOCAB:
            for tokens in TOKENS:
                try:
                    loss, step = hh.hh_head_sizes(hh.make_head_cfg(hidden, vocab, tokens, dtype))
                except hh.HHError as e:
                    assert e.code == hh.HH_ERR_UNSUPPORTED_SHAPE
                    continue
                seen += 1
                assert loss <= most_loss and step <= most_step, (hidden, vocab, tokens)
    assert seen > 200


def test_copies_of_x_count(dtype=hh.HH_BF16):
    """d and the copies of x each up to 2 GiB: far more than d and the scores."""
    step = hh.hh_head_sizes(hh.make_head_cfg(32768, 32704, 16383, dtype))[1]
    assert 4.5 * GIB < step <= 4.6 * GIB
