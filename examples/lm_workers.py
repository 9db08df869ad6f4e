#!/usr/bin/env python
"""K workers train a next-token model with CoCoD-SGD on one GPU, every gradient formed by the language-model operators.

    python examples/lm_workers.py [--workers 8] [--vocab 2048] [--width 512] [--rounds 60] [--optimizer adamw --lr 0.001 --bits 8]

The model: a fixed embedding of the token before, two ReLU layers, a vocabulary.  Every worker has weights and a mini-batch of
its own, of its own size (Algorithm 1's M_i).  One local step:

    forward    z = x w^T by worker (grouped_forward), ReLU, and the activation kept in 8 bits (act_pack)
    loss       softmax cross-entropy over the vocabulary and its gradient (vocab_loss_grad), straight into the K x P gradients
    backward   the ReLU's gate from the checkpoint (act_relu_grad), the weight gradient from the checkpoint
               (grouped_weight_grad), the gradient of the layer's input (grouped_input_grad)
    update     Engine.local_step on the K x P gradients, which also keeps the bf16 copy that the products read (or EngineAdamW.local_step)

and a round is k of them between comm_begin and comm_end.  The text is a Markov chain: every token is followed by one of four
others, so that no model gets below log 4 = 1.386.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1906_12043_b200 import engine as E, lm, optim  # noqa: E402

FOLLOWERS = 4


class Workers:
    def __init__(self, sizes, vocab, embed, width, lr, mu, seed=0, adamw_bits=0):
        """sizes: tokens in each worker's mini-batch.  adamw_bits: 0 (momentum SGD), or AdamW with its moments in 8 or 32 bits."""
        self.K, self.vocab, self.embed, self.width = len(sizes), vocab, embed, width
        self.shapes = [(width, embed), (width, width), (vocab, width)]
        self.starts, at = [], 0
        for n, k in self.shapes:
            self.starts.append(at)
            at += n * k
        self.P = -(-at // 64) * 64
        gen = torch.Generator().manual_seed(seed)
        x0 = torch.zeros(self.P)
        for (n, k), s in zip(self.shapes, self.starts):
            x0[s:s + n * k] = torch.randn(n * k, generator=gen) * (2.0 / k) ** 0.5
        self.table = torch.randint(0, vocab, (vocab, FOLLOWERS), generator=gen).cuda()
        self.embedding = torch.randn(vocab, embed, generator=gen).bfloat16().cuda()
        self.engine = E.Engine(self.K, self.P, lr, mu, 0.0)
        self.engine.set_option(E.OPT_BF16_SHADOW, 1)
        self.engine.set_params(x0.cuda())
        self.engine.set_batch_sizes([float(s) for s in sizes])
        self.local_step = self.engine.local_step
        if adamw_bits:
            self.opt = optim.EngineAdamW(self.engine, [(n * k, 0.01) for n, k in self.shapes], lr=lr, betas=(0.9, 0.95), state_bits=adamw_bits)
            self.local_step = self.opt.local_step
        self.ops = lm.LMOps()
        self.grads = torch.zeros(self.K, self.P, device="cuda")
        ends = torch.tensor([0] + list(sizes)).cumsum(0)
        self.offsets, self.tokens = ends.to(torch.int32).cuda(), int(ends[-1])
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 1)

    def views(self, flat):
        """The K workers' matrices in a K x P buffer."""
        return [flat[:, s:s + n * k].view(self.K, n, k) for (n, k), s in zip(self.shapes, self.starts)]

    def batch(self):
        before = torch.randint(0, self.vocab, (self.tokens,), generator=self.gen, device="cuda")
        which = torch.randint(0, FOLLOWERS, (self.tokens,), generator=self.gen, device="cuda")
        return before, self.table[before, which].to(torch.int32)

    def gradients(self, before, after):
        """The workers' gradients into self.grads; the workers' losses."""
        ops, off = self.ops, self.offsets
        w1, w2, w3 = self.views(self.engine.bf16_shadow())
        g1, g2, g3 = self.views(self.grads)
        x = self.embedding[before]
        kept1 = ops.act_pack(h := ops.grouped_forward(x, w1, off).relu_())
        kept2 = ops.act_pack(h := ops.grouped_forward(h, w2, off).relu_())
        loss, _, dh, _ = ops.vocab_loss_grad(h, w3, after, off, dw=g3)
        dz = ops.act_relu_grad(dh, kept2, out=dh)
        ops.grouped_weight_grad(dz, kept1, off, out=g2)
        dh = ops.grouped_input_grad(dz, w2, off)
        dz = ops.act_relu_grad(dh, kept1, out=dh)
        ops.grouped_weight_grad(dz, x, off, out=g1)
        return loss

    def round(self, k, side):
        """One round of Algorithm 1; the workers' losses at its k steps."""
        losses = []
        self.engine.comm_begin(side)
        for _ in range(k):
            losses.append(self.gradients(*self.batch()))
            self.local_step(self.grads)
        self.engine.comm_end()
        return torch.stack(losses)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=1024, help="tokens in a worker's mini-batch; every other worker has half of them")
    ap.add_argument("--vocab", type=int, default=2048)
    ap.add_argument("--embed", type=int, default=256)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--rounds", type=int, default=60)
    ap.add_argument("--k", type=int, default=4, help="local steps in a round")
    ap.add_argument("--lr", type=float, default=0.5)
    ap.add_argument("--optimizer", default="sgd", choices=("sgd", "adamw"))
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32), help="of AdamW's moments")
    a = ap.parse_args()
    sizes = [a.tokens // (1 + i % 2) for i in range(a.workers)]
    w = Workers(sizes, a.vocab, a.embed, a.width, a.lr, 0.9, adamw_bits=a.bits if a.optimizer == "adamw" else 0)
    side = torch.cuda.Stream(priority=-1)
    print(f"{a.workers} workers of {sum(n * k for n, k in w.shapes):,} parameters, {sum(sizes)} tokens a step")
    for r in range(a.rounds):
        losses = w.round(a.k, side)
        if r % 10 == 0 or r == a.rounds - 1:
            print(f"round {r:3d}: loss {losses.mean():.4f} (workers {losses[-1].min():.4f} .. {losses[-1].max():.4f})")
    w.ops.check()
    w.engine.sync()


if __name__ == "__main__":
    main()
