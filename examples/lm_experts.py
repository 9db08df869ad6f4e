#!/usr/bin/env python
"""A next-token model with mixtures of experts, every product, choice, gradient and update formed by the package's operators.

    python examples/lm_experts.py [--experts 16] [--top 2] [--layers 2] [--steps 200] [--bits 8]

The model: a fixed embedding of the token before, layers x <- x + sum over the chosen experts of p_e * W2_e relu(W1_e x), a vocabulary.  One step:

    router     logits = x R^T (grouped_forward), the top experts and their log probabilities (token_logprobs)
    experts    the tokens sorted by expert (expert_sort), their rows (expert_rows), two products by expert (grouped_forward) with the activation
               kept in 8 bits (act_pack), the weighted sum back (expert_join)
    loss       softmax cross-entropy over the vocabulary and its gradient (vocab_loss_grad)
    backward   expert_join_grad, the products' gradients, expert_rows_grad, and the router's through token_logprobs_grad
    update     AdamW over all tensors at once (optim.AdamW), moments in 8 bits or 32, which also writes the bf16 copies that the products read

and at the end the text is scored: log probabilities, entropy and alternatives from the logits (token_logprobs).  The text is a Markov chain: every
token is followed by one of four others, so that no model gets below log 4 = 1.386.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1906_12043_b200 import lm, optim  # noqa: E402

FOLLOWERS = 4


class Model:
    def __init__(self, vocab, width, hidden, experts, top, layers, lr, bits=8, seed=0):
        self.vocab, self.width, self.experts, self.top, self.layers = vocab, width, experts, top, layers
        gen = torch.Generator().manual_seed(seed)

        def weights(*shape):
            return (torch.randn(*shape, generator=gen) * shape[-1] ** -0.5).cuda()

        # router, first and second product of each layer, then the vocabulary: G x n x k, as the products by group take them
        self.params = [w for _ in range(layers) for w in (weights(1, experts, width), weights(experts, hidden, width), weights(experts, width, hidden))]
        self.params.append(weights(1, vocab, width))
        self.copies = [w.bfloat16() for w in self.params]
        self.opt = optim.AdamW(self.params, lr=lr, betas=(0.9, 0.95), weight_decay=[0.0 if w.shape[0] == 1 else 0.01 for w in self.params], state_bits=bits,
                               copies=self.copies)
        self.ops = lm.LMOps()
        self.table = torch.randint(0, vocab, (vocab, FOLLOWERS), generator=gen).cuda()
        self.embedding = torch.randn(vocab, width, generator=gen).bfloat16().cuda()
        self.gen = torch.Generator(device="cuda").manual_seed(seed + 1)

    def batch(self, tokens):
        before = torch.randint(0, self.vocab, (tokens,), generator=self.gen, device="cuda")
        which = torch.randint(0, FOLLOWERS, (tokens,), generator=self.gen, device="cuda")
        return before, self.table[before, which].to(torch.int32)

    def forward(self, before):
        """The last layer's output, and what the backward pass needs of each layer."""
        ops = self.ops
        x = self.embedding[before]
        whole = torch.arange(2, dtype=torch.int32, device="cuda") * len(before)
        kept = []
        for i in range(self.layers):
            router, w1, w2 = self.copies[3 * i:3 * i + 3]
            logits = ops.grouped_forward(x, router, whole)
            chosen = ops.token_logprobs(logits, top=self.top)
            plan = ops.expert_sort(chosen.top_tokens, self.experts)
            p = chosen.top_logp.exp()
            rows = ops.expert_rows(x, plan)
            h = ops.grouped_forward(rows, w1, plan.offsets).relu_()
            out = ops.grouped_forward(h, w2, plan.offsets)
            kept.append((x, logits, chosen, plan, p, rows, ops.act_pack(h), out))
            x = x + ops.expert_join(out, plan, p)
        return x, whole, kept

    def gradients(self, before, after):
        """(loss, the gradients of all parameters in float32)"""
        ops = self.ops
        x, whole, kept = self.forward(before)
        grads = [None] * len(self.params)
        loss, _, dx, grads[-1] = ops.vocab_loss_grad(x, self.copies[-1], after, whole, dw_dtype=torch.float32)
        for i in reversed(range(self.layers)):
            router, w1, w2 = self.copies[3 * i:3 * i + 3]
            x, logits, chosen, plan, p, rows, h, out = kept[i]
            dout, dp = ops.expert_join_grad(dx, out, plan, p)
            grads[3 * i + 2] = ops.grouped_weight_grad(dout, h, plan.offsets)
            dh = ops.act_relu_grad(ops.grouped_input_grad(dout, w2, plan.offsets), h)
            grads[3 * i + 1] = ops.grouped_weight_grad(dh, rows, plan.offsets)
            dlogits = ops.token_logprobs_grad(logits, None, chosen, d_top=dp * p)
            grads[3 * i] = ops.grouped_weight_grad(dlogits, x, whole)
            if i:
                dx = dx + ops.expert_rows_grad(ops.grouped_input_grad(dh, w1, plan.offsets), plan) + ops.grouped_input_grad(dlogits, router, whole)
        return loss, grads

    def step(self, before, after):
        loss, grads = self.gradients(before, after)
        self.opt.step(grads)
        return loss

    def score(self, before, after, top=FOLLOWERS):
        """Log probabilities of the tokens that follow, entropies and the most probable tokens."""
        x, whole, _ = self.forward(before)
        return self.ops.token_logprobs(self.ops.grouped_forward(x, self.copies[-1], whole), after, top=top)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--experts", type=int, default=16)
    ap.add_argument("--top", type=int, default=2)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=512)
    ap.add_argument("--vocab", type=int, default=2048)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    m = Model(a.vocab, a.width, a.hidden, a.experts, a.top, a.layers, a.lr, a.bits)
    print(f"{sum(p.numel() for p in m.params):,} parameters, {a.tokens} tokens a step, moments in {a.bits} bits")
    for s in range(a.steps):
        loss = m.step(*m.batch(a.tokens))
        if s % 20 == 0 or s == a.steps - 1:
            print(f"step {s:4d}: loss {float(loss):.4f}")
    before, after = m.batch(a.tokens)
    r = m.score(before, after)
    there = (r.top_tokens == after[:, None]).any(1).float().mean()
    print(f"scored: log probability {r.logp.mean():.4f}, entropy {r.entropy.mean():.4f}, the token among the first {FOLLOWERS}: {100 * there:.1f} %")
    m.ops.check()


if __name__ == "__main__":
    main()
