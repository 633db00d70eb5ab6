"""The tail of a last stage (final norm, residual projection in microscaled floating point with dropout): against its fp64 formula, and in
training steps of the stage."""
import json
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import mx_oracle as O
from paper_2405_16256_amd import binding as hh
from paper_2405_16256_amd import glue as L
from paper_2405_16256_amd import inputs as I
from paper_2405_16256_amd import last_stage as S

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHAPE = I.LayerShape(256, 4, 64, 320, 70, 1)


def oracle(t, y, dn, use, fmt, p, start):
    """-> forward's result and all gradients, of the tail's parameters; `start`: what the gradients hold before."""
    w = {n: L.to_np(v) for n, v in t.w.items()}
    eps = float(np.float32(1e-5))
    if fmt is None:
        dy, dg = O.norm_grad(y, w["g_norm"], eps, dn, 0.0)
        return O.norm(y, w["g_norm"], eps), dy, {"g_norm": dg + start}
    f = {"e4m3": O.E4M3, "e2m1": O.E2M1}[fmt]
    x = O.norm(y, w["g_proj"], eps)
    h = y + O.dropout(O.rounded(x, f) @ O.rounded(w["w_proj"], f).T, p, t.seed, use)
    dh, dg_norm = O.norm_grad(h, w["g_norm"], eps, dn, 0.0)
    d = O.dropout(dh, p, t.seed, use)
    dx = O.rounded(d, f) @ O.rounded(w["w_proj"].T, f).T
    dw = O.rounded(d.T, f) @ O.rounded(x.T, f).T
    dy, dg_proj = O.norm_grad(y, w["g_proj"], eps, dx, dh)
    return O.norm(h, w["g_norm"], eps), dy, {"g_norm": dg_norm + start, "g_proj": dg_proj + start, "w_proj": dw + start}


@pytest.mark.parametrize("bf16", (True, False))
@pytest.mark.parametrize("fmt,p", [(None, 0.0), ("e4m3", 0.0), ("e4m3", 0.25), ("e2m1", 0.5)])
def test_tail_against_its_formula(bf16, fmt, p):
    """fp32 storage: sums in fp32, and a value at a border between two numbers of a format may fall on the other side, a step of 2^-3 (E2M1: 2^-1) of
    that value: with one in 10^5 at such a border, 2^-3 / 300 of a tensor's norm.  bf16 storage: the library's tolerances of bf16, and what is
    packed was rounded to bf16 first, which moves every 2^8 / 2^4-th value (E2M1: 2^8 / 2^2) across a border."""
    ctx = hh.hh_ctx_create(0)
    t = S.make_tail(3, SHAPE, bf16, fmt, p)
    y, dn = I.activations(3, SHAPE, 0, bf16)
    y, dn = (v.reshape(SHAPE.tokens, SHAPE.hidden) for v in (y, dn))
    ws = torch.empty(t.workspace_bytes, dtype=torch.uint8, device=L.DEV)
    yd, dd = L.to_dev(y, bf16), L.to_dev(dn, bf16)
    dy = torch.empty_like(yd)
    t.pack(ctx, L.stream_ptr())
    for use, accumulate in ((5, False), (5, True)):
        n = t.forward(ctx, yd, use, ws, L.stream_ptr())
        start = 0.0
        if accumulate:
            for g in t.g.values():
                g.fill_(0.5)
            start = 0.5
        t.backward(ctx, yd, dd, dy, use, accumulate, ws, L.stream_ptr())
        torch.cuda.synchronize()
        want_n, want_dy, want_g = oracle(t, y.astype(np.float64), dn.astype(np.float64), use, fmt, p, start)
        tol = (2e-2, 5e-2) if bf16 else (1e-5, 1e-5) if fmt is None else (2e-3, 2e-3)
        errs = {"n": L.rel_err(L.to_np(n), want_n), "dy": L.rel_err(L.to_np(dy), want_dy)}
        errs.update({k: L.rel_err(L.to_np(t.g[k]), v) for k, v in want_g.items()})
        assert errs["n"] <= tol[0] and all(e <= tol[1] for e in errs.values()), errs
    assert set(want_g) == set(t.g)
    torch.cuda.synchronize()
    hh.hh_ctx_destroy(ctx)


def stage_of(bf16, tail, layers=1, vocab=300):
    head = I.normal(7, S.TID_HEAD, (vocab, SHAPE.hidden), scale=0.02)
    return S.LastStage(SHAPE, [I.layer_weights(7, l, SHAPE, bf16) for l in range(layers)], head, bf16, tail=tail)


def run(stage, bf16, steps):
    x, labels = S.batch(7, SHAPE, 300, 2, bf16)
    x, labels = [L.to_dev(t, bf16) for t in x], [torch.from_numpy(t).to(L.DEV) for t in labels]
    losses, dx = [torch.empty(SHAPE.tokens, device=L.DEV) for _ in x], [torch.empty_like(t) for t in x]
    for _ in range(steps):
        stage.gradients(x, labels, losses, dx)
        stage.update()
    torch.cuda.synchronize()
    return losses, dx


@pytest.mark.parametrize("bf16", (True, False))
@pytest.mark.parametrize("fmt,p", [(None, 0.0), ("e4m3", 0.25), ("e2m1", 0.0)])
def test_a_stage_with_a_tail_takes_steps(bf16, fmt, p):
    runs = []
    for _ in range(2):
        stage = stage_of(bf16, S.make_tail(7, SHAPE, bf16, fmt, p))
        before = {n: t.clone() for n, t in stage.tail.w.items()}
        losses, dx = run(stage, bf16, 3)
        assert stage.step_no == 3 and all(bool(torch.isfinite(t).all()) for t in losses + dx)
        assert all(bool(g.any()) for g in stage.tail.g.values()) and all(not torch.equal(before[n], t) for n, t in stage.tail.w.items())
        runs.append([t.clone() for t in losses + dx] + [p.clone() for p, _, _ in stage.params])
        stage.close()
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_what_is_dropped_differs_from_pass_to_pass():
    stage = stage_of(True, S.make_tail(7, SHAPE, True, "e4m3", 0.5))
    y, st = L.to_dev(I.activations(7, SHAPE, 0, True)[0], True), L.stream_ptr()
    sums = []
    for use in (0, 1, 0):
        stage.tail.forward(stage.ctx, y, use, stage.ws, st)
        sums.append(stage.tail.sum.clone())
    assert torch.equal(sums[0], sums[2]) and not torch.equal(sums[0], sums[1])
    x, _ = run(stage, True, 2)
    assert stage._passes == 4
    stage.close()


def test_a_tail_of_another_shape_is_refused():
    other = I.LayerShape(256, 4, 64, 320, 71, 1)
    for tail in (S.make_tail(7, other, True, None), S.make_tail(7, SHAPE, False, None)):
        with pytest.raises(ValueError):
            stage_of(True, tail)
    with pytest.raises(ValueError):
        S.Tail(70, 256, True, np.ones(256, dtype=np.float32), dropout=0.1)


@pytest.mark.parametrize("flags", (["--norm"], ["--project", "e4m3", "--dropout", "0.1"], ["--project", "e2m1", "--f32"]))
def test_command_runs(flags):
    out = subprocess.run([sys.executable, "-m", "paper_2405_16256_amd.last_stage", "--steps", "2", "--layers", "1", *flags], cwd=ROOT, capture_output=True, text=True,
                         timeout=100)
    assert out.returncode == 0, out.stderr
    lines = [json.loads(t) for t in out.stdout.splitlines()]
    assert [t["step"] for t in lines] == [0, 1] and all(np.isfinite(t["loss"]) and np.isfinite(t["grad_norm"]) for t in lines)
