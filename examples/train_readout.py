"""Fits a readout to a frozen model and decodes with it.

    python examples/train_readout.py [--shape tiny] [--tokens 1024] [--steps 60]

The frozen model (synthetic weights) runs over a stream of tokens; for every token
the residual after the readout's layer and the final one are kept.  The full
model's answers -- its best tokens with their log probabilities -- are the teacher.
The readout's matrix and offset start at identity and zero and are fitted by
distilling those answers through the model's own final norm and unembedding, both
frozen.  At the end an engine decodes with the fitted readout.

Everything but the optimiser's element-wise update runs in the library: `linear`,
`rms_norm`, `token_logprobs`, `distill_topk_step` and their backward passes.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_14144_gb300 as ee  # noqa: E402
import synth  # noqa: E402

BEST = 32  # teacher tokens per position


def bf16(bits: np.ndarray):
    """bf16 bit patterns of the synthetic weights as a CUDA tensor."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def bits(t) -> np.ndarray:
    return t.to(torch.bfloat16).cpu().view(torch.int16).numpy().view(np.uint16)


def residuals(shape, model, n: int):
    """Residuals after the readout's layer and after the last one, [n, d] each, of the
    full model over a stream of n tokens."""
    eng = ee.Engine(shape.replace(prompt_len=1, new_tokens=n + 1), model)
    ids = synth.calibration_stream(shape, n + 1)
    eng.prefill(ids[:1])
    at_readout = np.empty((n, shape.d_model), np.float32)
    final = np.empty_like(at_readout)
    for i in range(n):
        eng.decode_step(int(ids[i + 1]), None, ee.FORCE_FULL)
        at_readout[i], final[i] = eng.hidden_at_readout(0), eng.hidden_final()
    eng.close()
    return torch.from_numpy(at_readout).cuda(), torch.from_numpy(final).cuda()


class Readout:
    """y = h W^T + b in front of the frozen norm and unembedding, with Adam's state."""

    def __init__(self, d: int, gain, unembedding, eps: float):
        self.gain, self.unembedding, self.eps = gain, unembedding, eps
        # 32-bit masters, 16-bit copies for the products
        self.masters = [torch.eye(d, device="cuda"), torch.zeros(d, device="cuda")]
        self.m = [torch.zeros_like(p) for p in self.masters]
        self.v = [torch.zeros_like(p) for p in self.masters]
        self.t = 0

    def logits(self, h, keep: bool = False):
        w, b = (p.to(torch.bfloat16) for p in self.masters)
        y = ee.linear(h, w, b)
        z, rstd = ee.rms_norm(y, self.gain, self.eps)
        out = ee.linear(z, self.unembedding)
        return (out, y, rstd) if keep else out

    def step(self, h, ids, teacher, weight, lr: float):
        """One update on a batch; returns the loss of each row before it."""
        logits, y, rstd = self.logits(h, keep=True)
        # the gradient takes the logits' place
        loss, dlogits = ee.distill_topk_step(logits, ids, teacher, weight, tail=True, grad=logits)
        dz, _, _ = ee.linear_backward(dlogits, None, self.unembedding, dw=False, dbias=False)
        dy, _ = ee.rms_norm_backward(dz, y, self.gain, rstd, dgain=False)
        _, dw, db = ee.linear_backward(dy, h, None, dx=False, dw_dtype=torch.float32)
        self.t += 1
        for p, g, m, v in zip(self.masters, (dw, db), self.m, self.v):
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.999).addcmul_(g, g, value=0.001)
            p.sub_(lr * (m / (1 - 0.9 ** self.t)) / ((v / (1 - 0.999 ** self.t)).sqrt() + 1e-8))
        return loss


def fit(shape, model, tokens: int = 1024, steps: int = 60, lr: float = 1e-3, report=print) -> dict:
    h, final = residuals(shape, model, tokens)
    h = h.to(torch.bfloat16)
    gain = bf16(model["final_norm"])
    unembedding = bf16(model["embed"] if model["lm_head"] is None else model["lm_head"])
    # the teacher: the full model's best tokens and what it gives the rest
    z, _ = ee.rms_norm(final, gain, shape.rms_eps, out_dtype=torch.bfloat16)
    _, entropy, _, teacher, ids = ee.token_logprobs(ee.linear(z, unembedding), k=BEST)
    answers = ids[:, 0].contiguous()
    train = tokens * 3 // 4
    weight = torch.full((train,), 1.0 / train, device="cuda")
    ro = Readout(shape.d_model, gain, unembedding, shape.rms_eps)

    def score(rows):
        """Share of the full model's answers given, and their mean log probability."""
        lp, _, _, _, top = ee.token_logprobs(ro.logits(h[rows]), answers[rows], k=1)
        return (top[:, 0] == answers[rows]).float().mean().item(), lp.mean().item()

    parts = (("training", slice(0, train)), ("held out", slice(train, tokens)))
    before = {name: score(rows) for name, rows in parts}
    losses = []
    for i in range(steps):
        loss = ro.step(h[:train], ids[:train], teacher[:train], weight, lr)
        losses.append(loss.mean())
        if report and (i % 10 == 0 or i + 1 == steps):
            report(f"step {i:3d}  loss {losses[-1].item():.4f}")
    after = {name: score(rows) for name, rows in parts}
    if report:
        report(f"teacher's mean entropy {entropy.mean().item():.3f}")
        for name, _ in parts:
            report(f"{name}: answers {before[name][0]:.3f} -> {after[name][0]:.3f}, their log probability "
                   f"{before[name][1]:.3f} -> {after[name][1]:.3f}")
    fitted = dict(model)
    fitted["readouts"] = [(shape.readout_layers[0], bits(ro.masters[0]), bits(ro.masters[1]))]
    return {"model": fitted, "losses": [x.item() for x in losses], "before": before, "after": after}


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--shape", default="tiny", choices=sorted(synth.CONFIGS))
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=60)
    args = ap.parse_args()
    shape = synth.CONFIGS[args.shape]
    model = synth.make_model(shape)
    out = fit(shape, model, args.tokens, args.steps)
    for name, m in (("readout of the synthetic model", model), ("fitted readout", out["model"])):
        eng = ee.Engine(shape, m)
        eng.prefill(synth.prompt(shape))
        eng.decode_n(min(64, shape.new_tokens), taus=[0.5])
        st = eng.stats()
        print(f"{name}: {st['exits'][0]} of {st['steps']} tokens exit at tau 0.5")
        eng.close()


if __name__ == "__main__":
    main()
