"""Distilling a student's output head in 8 bits, committed step by committed step.

Each step runs, on one GPU:

  norm       the last layer's output added to the residual stream, normalised and
             quantized by rows and transposed (``apc.rms_norm_fp8``)
  quantize   the head's working copy in square blocks (``apc.quantize_fp8``)
  logits     their block-scaled 8-bit product (``apc.matmul_fp8``)
  loss       distillation from the teacher's largest logits, with the gradient
             written over the logits (``apc.distill_loss_grad``)
  backward   the gradient quantized both ways, and two more products: the norm's
             output's gradient and the head's; the norm's gradient
             (``apc.rms_norm_grad``)
  commit     the norm of all gradients (``apc.grad_norm``), AdamW on the fp32 masters
             and moments of head and norm with the gradients clipped by it, the new
             working copies and the digests of all four (``apc.commit_step``)

and does so for two replicas, whose digests have to agree after every step: no
operator's result depends on the order in which anything ran.  Data and weights are
random; the loss falls because the student learns the teacher.

    python examples/distill_head.py --steps 8
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2609_18178_gb300 as apc

TEMPERATURE, KD_WEIGHT, LABEL_WEIGHT = 2.0, 0.9, 0.1
EPS, MAX_NORM = 1e-5, 0.05
HPARAMS = dict(lr=2e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0)


class Head:
    """One replica: the master weights of head and norm, their moments, working
    copies and gradients."""

    def __init__(self, vocab: int, hidden: int):
        gen = torch.Generator(device="cuda").manual_seed(0)
        self.p = torch.randn(vocab, hidden, generator=gen, device="cuda").mul_(0.02)
        self.scale = torch.ones(hidden, device="cuda")
        self.w, self.scale_w = self.p.bfloat16(), self.scale.bfloat16()
        self.g, self.scale_g = torch.empty_like(self.w), torch.empty_like(self.scale_w)
        at = 0
        table = []
        for p, g, w in ((self.p, self.g, self.w), (self.scale, self.scale_g, self.scale_w)):
            table.append(apc.TensorEntry(p, torch.zeros_like(p), torch.zeros_like(p), g, w, at))
            at += p.numel()
        self.table = apc.prepare_table(table)

    def step(self, x, residual, ids, teacher, labels, weights, t: int):
        """One committed step; the positions' losses, the gradient of x and
        residual, the gradients' norm and the digests of p, m, v and w."""
        x8, xs, x8t, xst, h, rstd = apc.rms_norm_fp8(x, self.scale_w, eps=EPS, residual=residual, transposed=True)
        w8, ws, w8t, wst = apc.quantize_fp8(self.w, block_rows=128, transposed=True)
        logits = apc.matmul_fp8(x8, xs, w8, ws)
        loss, _, d = apc.distill_loss_grad(logits, ids, teacher, weights, temperature=TEMPERATURE, kd_weight=KD_WEIGHT,
                                           labels=labels, label_weight=LABEL_WEIGHT, out=logits)
        d8, ds, d8t, dst = apc.quantize_fp8(d, transposed=True)
        dy = apc.matmul_fp8(d8, ds, w8t, wst)                        # [tokens, hidden]
        apc.matmul_fp8(d8t, dst, x8t, xst, out=self.g)               # [vocab, hidden]
        dx, _ = apc.rms_norm_grad(dy, h, self.scale_w, rstd, out=dy, dweight=self.scale_g)
        norm = apc.grad_norm(self.table)
        return loss, dx, norm, apc.commit_step(self.table, t, HPARAMS, grad_norm=norm, max_norm=MAX_NORM)


def main(argv=None) -> list:
    """Runs the steps; the mean loss after each."""
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--tokens", type=int, default=1024)
    a.add_argument("--vocab", type=int, default=32768)
    a.add_argument("--hidden", type=int, default=4096)
    a.add_argument("--k", type=int, default=64)
    a.add_argument("--steps", type=int, default=8)
    a = a.parse_args(argv)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, residual = (torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16() for _ in range(2))
    # a teacher's head near the student's start, its k largest logits
    target = torch.randn(a.vocab, a.hidden, generator=gen, device="cuda").mul_(0.04).bfloat16()
    y, _, _ = apc.rms_norm(x, torch.ones(a.hidden, device="cuda"), eps=EPS, residual=residual)
    teacher, ids = (y @ target.t()).float().topk(a.k, 1)
    labels = ids[:, 0].contiguous()
    weights = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")
    replicas = [Head(a.vocab, a.hidden) for _ in range(2)]
    losses = []
    for t in range(1, a.steps + 1):
        out = [r.step(x, residual, ids, teacher, labels, weights, t) for r in replicas]
        digests = [apc.digests_to_host(o[3]) for o in out]
        if digests[0] != digests[1]:
            raise RuntimeError("step %d: the replicas' states differ: %s" % (t, digests))
        losses.append(float(out[0][0].mean()))
        print("step %d: loss %.4f, |dx| %.3g, |g| %.3g, digests %s" % (t, losses[-1], float(out[0][1].float().norm()), float(out[0][2]),
                                                                       " ".join("%016x" % d for d in digests[0])))
    if apc.device_status():
        raise RuntimeError("a bounded wait gave up")
    return losses


if __name__ == "__main__":
    main()
