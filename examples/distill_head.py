"""Distilling a student's output head in 8 bits, committed step by committed step.

Each step runs, on one GPU:

  quantize   the activations by rows and transposed, the head's working copy in
             square blocks (``apc.quantize_fp8``)
  logits     their block-scaled 8-bit product (``apc.matmul_fp8``)
  loss       distillation from the teacher's largest logits, with the gradient
             written over the logits (``apc.distill_loss_grad``)
  backward   the gradient quantized both ways, and two more products: the
             activations' gradient and the head's
  commit     AdamW on the head's fp32 master and moments, its new working copy and
             the digests of all four (``apc.commit_step``)

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
HPARAMS = dict(lr=2e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.0)


class Head:
    """One replica: the head's master weights, moments and working copy."""

    def __init__(self, vocab: int, hidden: int):
        gen = torch.Generator(device="cuda").manual_seed(0)
        self.p = torch.randn(vocab, hidden, generator=gen, device="cuda").mul_(0.02)
        self.m, self.v = torch.zeros_like(self.p), torch.zeros_like(self.p)
        self.w = self.p.bfloat16()
        self.g = torch.empty_like(self.w)

    def step(self, x, ids, teacher, labels, weights, t: int):
        """One committed step; the positions' losses, the activations' gradient
        and the digests of p, m, v and w."""
        x8, xs, x8t, xst = apc.quantize_fp8(x, transposed=True)
        w8, ws, w8t, wst = apc.quantize_fp8(self.w, block_rows=128, transposed=True)
        logits = apc.matmul_fp8(x8, xs, w8, ws)
        loss, _, d = apc.distill_loss_grad(logits, ids, teacher, weights, temperature=TEMPERATURE, kd_weight=KD_WEIGHT,
                                           labels=labels, label_weight=LABEL_WEIGHT, out=logits)
        d8, ds, d8t, dst = apc.quantize_fp8(d, transposed=True)
        dx = apc.matmul_fp8(d8, ds, w8t, wst)                        # [tokens, hidden]
        apc.matmul_fp8(d8t, dst, x8t, xst, out=self.g)               # [vocab, hidden]
        digests = apc.commit_step([apc.TensorEntry(self.p, self.m, self.v, self.g, self.w)], t, HPARAMS)
        return loss, dx, digests


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
    x = torch.randn(a.tokens, a.hidden, generator=gen, device="cuda").bfloat16()
    # a teacher's head near the student's start, its k largest logits
    target = torch.randn(a.vocab, a.hidden, generator=gen, device="cuda").mul_(0.04).bfloat16()
    teacher, ids = (x @ target.t()).float().topk(a.k, 1)
    labels = ids[:, 0].contiguous()
    weights = torch.full((a.tokens,), 1.0 / a.tokens, device="cuda")
    replicas = [Head(a.vocab, a.hidden) for _ in range(2)]
    losses = []
    for t in range(1, a.steps + 1):
        out = [r.step(x, ids, teacher, labels, weights, t) for r in replicas]
        digests = [apc.digests_to_host(o[2]) for o in out]
        if digests[0] != digests[1]:
            raise RuntimeError("step %d: the replicas' states differ: %s" % (t, digests))
        losses.append(float(out[0][0].mean()))
        print("step %d: loss %.4f, |dx| %.3g, digests %s" % (t, losses[-1], float(out[0][1].float().norm()),
                                                             " ".join("%016x" % d for d in digests[0])))
    if apc.device_status():
        raise RuntimeError("a bounded wait gave up")
    return losses


if __name__ == "__main__":
    main()
