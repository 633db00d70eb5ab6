"""Training of a pipeline's last stage on one device (Section 2.3 of the paper: the last stage turns its layers' output into a
loss before its backward pass can begin, and every device ends a step by applying the gradients of all micro-batches).

    hh_layer_fwd x layers -> hh_head_step -> hh_layer_bwd x layers      for each micro-batch
    hh_grad_clip over all gradients, hh_adamw_step with its factor      once a step

``LastStage`` holds parameters, fp32 master copies, moments and gradients (bf16 or fp32 storage) and runs such steps; as a
command it trains on one fixed seeded batch and prints a JSON line a step: the loss falls, because the batch is learnt.  The
output projection reads the layers' output as it is, or what a ``Tail`` (tail.py) makes of it: its norm, or that of its sum with a projection
in microscaled floating point.

  python -m paper_2405_16256_amd.last_stage [--steps 20] [--layers 2] [--micro 2] [--vocab 1000] [--f32]
                                            [--norm] [--project e4m3|e2m1 [--dropout 0.1]]
"""
from __future__ import annotations

import argparse
import json

import numpy as np
import torch

from . import binding as hh
from . import glue as L
from . import inputs as I
from .tail import FORMATS, Tail

TID_HEAD, TID_LABELS, TID_TAIL = 5, 6, 7   # tensor ids of the output projection, of the labels and of the tail's parameters (7, 8, 9)


class LastStage:
    """``s``: shape of a layer and its micro-batch; ``weights``: a dict of arrays a layer (inputs.layer_weights); ``head``: [vocab, hidden];
    ``tail``: a Tail of the same tokens, width and type, or None."""

    def __init__(self, s: I.LayerShape, weights, head: np.ndarray, bf16: bool, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, decay=0.1,
                 max_norm=1.0, tail: Tail | None = None):
        self.s, self.lr, self.betas, self.eps, self.max_norm = s, lr, (beta1, beta2), eps, max_norm
        dt = torch.bfloat16 if bf16 else torch.float32
        self.ctx, self.cfg = hh.hh_ctx_create(0), L.cfg_of(s, bf16)
        self.layers = [L.DeviceLayer(w, s, bf16) for w in weights]
        self.head = L.to_dev(head, bf16)
        self.dhead = torch.zeros(head.shape, dtype=torch.float32, device=L.DEV)
        self.head_cfg = hh.make_head_cfg(s.hidden, head.shape[0], s.tokens, hh.HH_BF16 if bf16 else hh.HH_F32)
        # every parameter with its gradient; norm gains have no weight decay
        self.params = [(l.w[n], l.g[n], 0.0 if n.startswith("g_") else decay) for l in self.layers for n in hh.WEIGHT_FIELDS]
        self.params.append((self.head, self.dhead, decay))
        self.tail, self._passes = tail, 0
        if tail is not None:
            if (tail.tokens, tail.hidden, tail.dtype) != (s.tokens, s.hidden, self.head_cfg.dtype):
                raise ValueError("the tail is of another shape or type than the stage")
            self.params += [(tail.w[n], tail.g[n], 0.0 if n.startswith("g_") else decay) for n in tail.w]
            tail.pack(self.ctx, L.stream_ptr())
        self.masters = [p.float() if bf16 else None for p, _, _ in self.params]
        self.moments = [(torch.zeros(p.shape, device=L.DEV), torch.zeros(p.shape, device=L.DEV)) for p, _, _ in self.params]
        self.clips = hh.make_clip_tensors([(g, None) for _, g, _ in self.params])
        self.updates = hh.make_adamw_tensors([(p, master, m, v, g, d) for (p, g, d), master, (m, v) in zip(self.params, self.masters, self.moments)])
        saved, ws = hh.hh_layer_sizes(self.cfg)
        ws = max(ws, hh.hh_head_sizes(self.head_cfg)[1], hh.HH_CLIP_WORKSPACE_BYTES, tail.workspace_bytes if tail is not None else 0)
        self.ws = torch.empty(ws, dtype=torch.uint8, device=L.DEV)
        self.saved = [torch.empty(saved, dtype=torch.uint8, device=L.DEV) for _ in self.layers]
        shape = (s.micro_batch, s.seq, s.hidden)
        self.acts = [torch.empty(shape, dtype=dt, device=L.DEV) for _ in self.layers]
        self.result = torch.empty(2, dtype=torch.float32, device=L.DEV)
        self.dloss = torch.empty(s.tokens, dtype=torch.float32, device=L.DEV)   # of each token's loss: one over the tokens that count

        # updates that changed the parameters: one whose factor is not finite leaves them alone and does not count
        self._applied, self._told, self._known = 0, torch.empty(2, dtype=torch.float32, pin_memory=True), None

    @property
    def step_no(self) -> int:
        """Updates applied so far; waits for the norm of the last one."""
        if self._known is not None:
            self._known.synchronize()
            self._applied += bool(torch.isfinite(self._told[1]))
            self._known = None
        return self._applied

    def close(self) -> None:
        torch.cuda.synchronize()
        hh.hh_ctx_destroy(self.ctx)

    def gradients(self, x, labels, losses, dx) -> None:
        """Loss of each token into losses[m] and the gradients of their mean, summed over the micro-batches; dx[m] [B, S, H] is what
        the stage before receives.  labels[m]: int64, negative where a token does not count; one past the vocabulary does not count either,
        and its loss is NaN.  Tokens are counted on the device: nothing here waits for it."""
        st = L.stream_ptr()
        counted = sum((((t >= 0) & (t < self.head.shape[0])).sum() for t in labels), torch.zeros((), dtype=torch.int64, device=L.DEV))
        self.dloss.copy_((1.0 / counted.clamp(min=1).double()).expand_as(self.dloss))
        for m in range(len(x)):
            ins = [x[m]] + self.acts[:-1]
            for layer, a, y, saved in zip(self.layers, ins, self.acts, self.saved):
                hh.hh_layer_fwd(self.ctx, self.cfg, layer.wstruct, a, y, saved, self.ws, st)
            last = self.acts[-1] if self.tail is None else self.tail.forward(self.ctx, self.acts[-1], self._passes, self.ws, st)
            hh.hh_head_step(self.ctx, self.head_cfg, last, self.head, labels[m], self.dloss, 1.0, losses[m], dx[m], self.dhead, m > 0,
                            self.ws, st)
            if self.tail is not None:
                self.tail.backward(self.ctx, self.acts[-1], dx[m], dx[m], self._passes, m > 0, self.ws, st)
            self._passes += 1
            for layer, a, saved in reversed(list(zip(self.layers, ins, self.saved))):
                hh.hh_layer_bwd(self.ctx, self.cfg, layer.wstruct, a, saved, dx[m], dx[m], layer.gstruct, m > 0, self.ws, st)

    def update(self) -> None:
        """Norm and factor of all gradients into self.result, then the clipped update.  The update's number in Adam's corrections depends on
        whether the one before was applied, so this waits for that one's norm, behind which the device has this step's gradients to do."""
        step = self.step_no + 1
        st = L.stream_ptr()
        hh.hh_grad_clip(self.ctx, self.clips, self.max_norm, self.result, self.ws, st)
        self._told.copy_(self.result, non_blocking=True)
        self._known = torch.cuda.Event()
        self._known.record()
        hh.hh_adamw_step(self.ctx, hh.make_adamw_cfg(self.lr, *self.betas, self.eps, step), self.updates, self.result[1:], st)
        if self.tail is not None:
            self.tail.pack(self.ctx, st)


def batch(seed: int, s: I.LayerShape, vocab: int, micro: int, bf16: bool):
    """Seeded boundary activations, and labels of which every eighth does not count."""
    x = [I.activations(seed, s, m, bf16)[0] for m in range(micro)]
    labels = []
    for m in range(micro):
        u = I.normal(seed, TID_LABELS + (m << 32), (s.tokens,))
        t = np.floor(np.abs(u) * 1e6).astype(np.int64) % vocab
        t[::8] = -100
        labels.append(t)
    return x, labels


def make_tail(seed: int, s: I.LayerShape, bf16: bool, project: str | None, dropout: float = 0.0) -> Tail:
    """A tail of seeded parameters."""
    g_norm, g_proj = (I.normal(seed, TID_TAIL + i, (s.hidden,), scale=0.02, mean=1.0) for i in range(2))
    if project is None:
        return Tail(s.tokens, s.hidden, bf16, g_norm)
    w = I.normal(seed, TID_TAIL + 2, (s.hidden, s.hidden), scale=0.02)
    return Tail(s.tokens, s.hidden, bf16, g_norm, g_proj, w, project, dropout, seed)


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--micro", type=int, default=2)
    ap.add_argument("--vocab", type=int, default=1000)
    ap.add_argument("--f32", action="store_true")
    ap.add_argument("--norm", action="store_true", help="a norm in front of the output projection")
    ap.add_argument("--project", choices=sorted(FORMATS), help="the same, and a residual projection in this format in front of it")
    ap.add_argument("--dropout", type=float, default=0.0, help="share of the projection's result that is dropped")
    a = ap.parse_args()
    if a.dropout and not a.project:
        ap.error("--dropout needs --project")
    bf16, seed = not a.f32, 7
    s = I.LayerShape(256, 4, 64, 704, 128, 1)
    head = I.normal(seed, TID_HEAD, (a.vocab, s.hidden), scale=0.02)
    tail = make_tail(seed, s, bf16, a.project, a.dropout) if a.norm or a.project else None
    stage = LastStage(s, [I.layer_weights(seed, l, s, bf16) for l in range(a.layers)], head, bf16, tail=tail)
    x, labels = batch(seed, s, a.vocab, a.micro, bf16)
    x = [L.to_dev(t, bf16) for t in x]
    labels = [torch.from_numpy(t).to(L.DEV) for t in labels]
    losses = [torch.empty(s.tokens, device=L.DEV) for _ in x]
    dx = [torch.empty_like(t) for t in x]
    counted = sum(int((t >= 0).sum()) for t in labels)
    for step in range(a.steps):
        stage.gradients(x, labels, losses, dx)
        stage.update()
        loss = sum(float(t.sum()) for t in losses) / counted
        norm, factor = stage.result.tolist()
        print(json.dumps({"step": step, "loss": round(loss, 5), "grad_norm": round(norm, 5), "clip_factor": round(factor, 5)}), flush=True)
    stage.close()


if __name__ == "__main__":
    main()
