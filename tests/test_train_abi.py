"""hh_train.h: host-side sizes, and refusals before any GPU work.  Runs without a GPU."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2405_16256_amd import binding as hh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, ODD = 1 << 20, (1 << 20) + 2          # addresses: aligned, aligned to two bytes


def test_structs_are_those_of_the_header(tmp_path):
    """The header is C, and the binding's structs have its fields' places."""
    structs = {n: getattr(hh, n) for n in ("hh_head_cfg", "hh_clip_tensor", "hh_adamw_tensor", "hh_adamw_cfg")}
    lines = ["#include <stdio.h>", '#include "hh_train.h"', "int main(void) {"]
    for n, s in structs.items():
        lines.append('printf("%s %%zu", sizeof(%s));' % (n, n))
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (n, f) for f, _ in s._fields_] + ['printf("\\n");']
    lines += ['printf("clip %zu\\n", HH_CLIP_WORKSPACE_BYTES); return 0; }']
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(line.split(" ", 1) for line in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for n, s in structs.items():
        assert [int(t) for t in out[n].split()] == [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_], n
    assert int(out["clip"]) == hh.HH_CLIP_WORKSPACE_BYTES


def head(**kw):
    d = dict(hidden=4096, vocab=32000, tokens=2048, dtype=hh.HH_BF16)
    d.update(kw)
    return hh.make_head_cfg(**d)


def test_head_sizes():
    loss, step = hh.hh_head_sizes(head())
    assert loss == 8 * 500 * 2048 + 4 * 2048                       # statistics of 500 slots a row, and the labels' scores
    d, xs = 4 * 2048 * 32000, 4 * 2048 * 4096
    assert d + xs < step < d + xs + (1 << 28) + (64 << 20) + 2 * loss
    # the workspace of a step is bounded however many tokens there are, and d never reaches 2^31 bytes
    assert hh.hh_head_sizes(head(tokens=200000))[1] < 3 << 30
    assert hh.hh_head_sizes(head(vocab=262144, hidden=64, tokens=1 << 20))[1] < 3 << 30
    assert hh.hh_head_sizes(head(dtype=hh.HH_F32))[0] >= 4 * 2048 * 32000
    loss_only = C.c_size_t()
    assert hh.lib.hh_head_sizes(C.byref(head()), C.byref(loss_only), None) == hh.HH_OK and loss_only.value == loss


BAD_HEAD = [(dict(hidden=0), hh.HH_ERR_INVALID_ARG), (dict(vocab=0), hh.HH_ERR_INVALID_ARG), (dict(tokens=0), hh.HH_ERR_INVALID_ARG),
            (dict(tokens=-3), hh.HH_ERR_INVALID_ARG), (dict(dtype=2), hh.HH_ERR_INVALID_ARG), (dict(hidden=4100), hh.HH_ERR_UNSUPPORTED_SHAPE),
            (dict(hidden=4, dtype=hh.HH_F32), hh.HH_ERR_UNSUPPORTED_SHAPE), (dict(hidden=32832), hh.HH_ERR_UNSUPPORTED_SHAPE),
            (dict(vocab=262145, hidden=64), hh.HH_ERR_UNSUPPORTED_SHAPE), (dict(tokens=262144), hh.HH_ERR_UNSUPPORTED_SHAPE),
            (dict(vocab=262144, hidden=8192), hh.HH_ERR_UNSUPPORTED_SHAPE), (dict(vocab=262144, hidden=4096, dtype=hh.HH_F32), hh.HH_ERR_UNSUPPORTED_SHAPE)]


@pytest.mark.parametrize("kw,code", BAD_HEAD)
def test_head_refuses_shapes(kw, code):
    cfg = head(**kw)
    for call in (lambda: hh.hh_head_sizes(cfg), lambda: hh.hh_head_loss(None, cfg, A, A, A, A, A),
                 lambda: hh.hh_head_step(None, cfg, A, A, A, None, 1.0, A, A, A, 0, A)):
        with pytest.raises(hh.HHError) as e:
            call()
        assert e.value.code == code and hh.hh_last_error()


def test_head_refuses_pointers():
    cfg = head()
    good = dict(x=A, w=A, labels=A, loss=A, workspace=A)
    for name in good:
        for p, code in ((None, hh.HH_ERR_INVALID_ARG), (ODD, hh.HH_ERR_MISALIGNED)):
            with pytest.raises(hh.HHError) as e:
                hh.hh_head_loss(None, cfg, **{**good, name: p})
            assert e.value.code == code and name in str(e.value)
    good = dict(good, dloss=None, scale=1.0, dx=A, dw=A, accumulate=0)
    for name in ("x", "w", "labels", "loss", "dx", "dw", "workspace", "dloss"):
        for p, code in ((None, hh.HH_ERR_INVALID_ARG), (ODD, hh.HH_ERR_MISALIGNED)):
            with pytest.raises(hh.HHError) as e:
                hh.hh_head_step(None, cfg, **{**good, name: p})
            assert e.value.code == (hh.HH_ERR_INVALID_ARG if p is None else code)
            assert name in str(e.value) or (name == "dloss" and p is None and "ctx" in str(e.value))   # dloss may be missing
    assert hh.lib.hh_head_loss(None, None, A, A, A, A, A, None) == hh.HH_ERR_INVALID_ARG
    assert hh.lib.hh_head_sizes(None, None, None) == hh.HH_ERR_INVALID_ARG


def test_shares_refuse():
    cfg = head()
    for call, good in ((hh.hh_head_share_fwd, dict(x=A, w=A, labels=A, lse=A, picked=A, workspace=A)),
                       (hh.hh_head_share_bwd, dict(x=A, w=A, labels=A, lse=A, dloss=None, scale=1.0, dx=A, dw=A, accumulate=0, workspace=A))):
        for name in good:
            if name in ("scale", "accumulate"):
                continue
            for p, code in ((None, hh.HH_ERR_INVALID_ARG), (ODD, hh.HH_ERR_MISALIGNED)):
                with pytest.raises(hh.HHError) as e:
                    call(None, cfg, first=0, **{**good, name: p})
                assert e.value.code == code
                assert name in str(e.value) or (name == "dloss" and p is None and "ctx" in str(e.value))
        for first in (-1, 2 ** 31 - 32000):
            with pytest.raises(hh.HHError) as e:
                call(None, cfg, first=first, **good)
            assert e.value.code == hh.HH_ERR_INVALID_ARG and "first" in str(e.value)
        with pytest.raises(hh.HHError) as e:
            call(None, head(hidden=100), first=0, **good)
        assert e.value.code == hh.HH_ERR_UNSUPPORTED_SHAPE


def clip_list(**kw):
    d = dict(g=A, out=A, count=5, dtype=hh.HH_F32)
    d.update(kw)
    return (hh.hh_clip_tensor * 1)(hh.hh_clip_tensor(**d))


@pytest.mark.parametrize("kw,code", [(dict(g=None), hh.HH_ERR_INVALID_ARG), (dict(g=ODD), hh.HH_ERR_MISALIGNED), (dict(out=ODD), hh.HH_ERR_MISALIGNED),
                                     (dict(dtype=2), hh.HH_ERR_INVALID_ARG), (dict(count=-1), hh.HH_ERR_INVALID_ARG), (dict(count=1 << 41), hh.HH_ERR_INVALID_ARG),
                                     (dict(dtype=hh.HH_BF16, g=A + 1), hh.HH_ERR_MISALIGNED)])
def test_clip_refuses_tensors(kw, code):
    with pytest.raises(hh.HHError) as e:
        hh.hh_grad_clip(None, clip_list(**kw), 1.0, A, A)
    assert e.value.code == code and "tensors[0]" in str(e.value)


def test_clip_refuses_the_rest():
    for args in ((clip_list(), 0.0, A, A), (clip_list(), -1.0, A, A), (clip_list(), float("nan"), A, A), (clip_list(), 1.0, None, A), (clip_list(), 1.0, A, None),
                 (clip_list(), 1.0, A, A), (clip_list(count=0, g=None, out=None), 1.0, A, A)):   # the last two: no context
        with pytest.raises(hh.HHError) as e:
            hh.hh_grad_clip(None, *args)
        assert e.value.code == hh.HH_ERR_INVALID_ARG
    with pytest.raises(hh.HHError) as e:
        hh.hh_grad_clip(None, clip_list(), 1.0, ODD, A)
    assert e.value.code == hh.HH_ERR_MISALIGNED
    assert hh.lib.hh_grad_clip(None, -1, clip_list(), 1.0, A, A, None) == hh.HH_ERR_INVALID_ARG
    assert hh.lib.hh_grad_clip(None, 1, None, 1.0, A, A, None) == hh.HH_ERR_INVALID_ARG


def adamw_list(**kw):
    d = dict(param=A, master=None, m=A, v=A, g=A, count=5, decay=0.1, param_dtype=hh.HH_F32, grad_dtype=hh.HH_F32)
    d.update(kw)
    return (hh.hh_adamw_tensor * 1)(hh.hh_adamw_tensor(**d))


@pytest.mark.parametrize("kw,code", [(dict(param=None), hh.HH_ERR_INVALID_ARG), (dict(m=None), hh.HH_ERR_INVALID_ARG), (dict(v=None), hh.HH_ERR_INVALID_ARG),
                                     (dict(g=None), hh.HH_ERR_INVALID_ARG), (dict(param=ODD), hh.HH_ERR_MISALIGNED), (dict(m=ODD), hh.HH_ERR_MISALIGNED),
                                     (dict(v=ODD), hh.HH_ERR_MISALIGNED), (dict(g=ODD), hh.HH_ERR_MISALIGNED), (dict(master=A), hh.HH_ERR_INVALID_ARG),
                                     (dict(param_dtype=hh.HH_BF16), hh.HH_ERR_INVALID_ARG), (dict(param_dtype=hh.HH_BF16, master=ODD), hh.HH_ERR_MISALIGNED),
                                     (dict(grad_dtype=7), hh.HH_ERR_INVALID_ARG), (dict(count=-1), hh.HH_ERR_INVALID_ARG), (dict(decay=-0.1), hh.HH_ERR_INVALID_ARG),
                                     (dict(decay=float("nan")), hh.HH_ERR_INVALID_ARG)])
def test_update_refuses_tensors(kw, code):
    with pytest.raises(hh.HHError) as e:
        hh.hh_adamw_step(None, hh.make_adamw_cfg(1e-3), adamw_list(**kw))
    assert e.value.code == code and "tensors[0]" in str(e.value)


@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(lr=1e-3, beta1=1.0), dict(lr=1e-3, beta2=-0.1), dict(lr=1e-3, eps=-1.0), dict(lr=1e-3, step=0),
                                dict(lr=float("nan")), dict(lr=1e-3, beta1=float("nan"))])
def test_update_refuses_settings(kw):
    with pytest.raises(hh.HHError) as e:
        hh.hh_adamw_step(None, hh.make_adamw_cfg(**kw), adamw_list())
    assert e.value.code == hh.HH_ERR_INVALID_ARG


def test_update_refuses_the_rest():
    assert hh.lib.hh_adamw_step(None, None, 1, adamw_list(), None, None) == hh.HH_ERR_INVALID_ARG
    cfg = hh.make_adamw_cfg(1e-3)
    assert hh.lib.hh_adamw_step(None, C.byref(cfg), 1, None, None, None) == hh.HH_ERR_INVALID_ARG
    assert hh.lib.hh_adamw_step(None, C.byref(cfg), -1, adamw_list(), None, None) == hh.HH_ERR_INVALID_ARG
    assert hh.lib.hh_adamw_step(None, C.byref(cfg), 1, adamw_list(), ODD, None) == hh.HH_ERR_MISALIGNED
    assert hh.lib.hh_adamw_step(None, C.byref(cfg), 1, adamw_list(), None, None) == hh.HH_ERR_INVALID_ARG and "ctx" in hh.hh_last_error()


def test_lists_refuse_what_does_not_go_together():
    f, b = torch.zeros(6), torch.zeros(6, dtype=torch.bfloat16)
    for pairs in ([(f.to(torch.float16), None)],):
        with pytest.raises(TypeError):
            hh.make_clip_tensors(pairs)
    with pytest.raises(TypeError):
        hh.make_clip_tensors([(f, b)])
    with pytest.raises(ValueError):
        hh.make_clip_tensors([(f, torch.zeros(5))])
    with pytest.raises(ValueError):
        hh.make_clip_tensors([(torch.zeros(4, 6).t(), None)])
    with pytest.raises(ValueError):
        hh.make_adamw_tensors([(f, None, f, f, f[:5], 0.0)])
    with pytest.raises(TypeError):
        hh.make_adamw_tensors([(b, f, b, f, f, 0.0)])
    with pytest.raises(TypeError):
        hh.make_adamw_tensors([(b, b, f, f, f, 0.0)])
    one = hh.make_adamw_tensors([(b, f, f, f, b, 0.5)])[0]
    assert (one.count, one.param_dtype, one.grad_dtype, one.decay) == (6, hh.HH_BF16, hh.HH_BF16, 0.5)
