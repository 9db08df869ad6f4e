"""Workloads of the language-model operators: what is measured, on which sizes and inputs.

Three operators, all over rows that belong to groups (the workers' mini-batches, of unequal sizes, or experts):

* products with each group's own weights: forward, gradient of the input, gradient of the weights;
* activation checkpoints held in 8 bits, and the two things a backward pass does with them (the gate of a ReLU, the
  gradient of the next layer's weights);
* softmax cross-entropy over a large vocabulary, with or without its gradient.

``run`` computes them in a plain form (32-bit torch operations, rounded once at the end), or, with ``own`` set, through
the package.
"""
import math
import random

import torch

own = False

IGNORED = -1          # label of a row that takes no part
BLOCK = 128           # columns that share a scale in an 8-bit checkpoint


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a handful of tokens over four experts, one of them idle: the call's own cost is what counts
        dict(name="forward, few rows", op="forward", groups=4, rows=24, n=512, k=512, out="bf16"),
        # the framework's 16 workers with mini-batches of unequal size (128 on average), the first layer of its MLP
        dict(name="forward, 16 workers", op="forward", groups=16, rows=2048, n=1024, k=784, out="bf16"),
        # the way back through a wide layer, an odd number of rows and a width that ends inside a tile
        dict(name="input gradient, odd sizes", op="input_grad", groups=5, rows=8191, n=4096, k=2040, out="bf16"),
        # gradients of large per-group weights, written as the fp32 matrix that the local step takes
        dict(name="weight gradient, large", op="weight_grad", groups=8, rows=16384, n=4096, k=2048, out="f32"),
        # a layer's activations go to 8 bits and come back
        dict(name="checkpoint and back", op="act_roundtrip", groups=1, rows=8191, n=0, k=4096, out="bf16"),
        # the gate of a ReLU from the checkpoint of a few rows, columns that end inside a block
        dict(name="gate from checkpoint, few rows", op="act_relu_grad", groups=1, rows=77, n=0, k=1000, out="bf16"),
        # the 16 workers' hidden layer: weight gradient from 8-bit activations
        dict(name="weight gradient from checkpoint", op="act_weight_grad", groups=16, rows=2048, n=1024, k=1024, out="f32"),
        # the same for long batches
        dict(name="weight gradient from checkpoint, large", op="act_weight_grad", groups=4, rows=32768, n=2048, k=4096, out="bf16"),
        # evaluation: the loss alone, odd vocabulary
        dict(name="vocabulary loss", op="vocab_loss", groups=1, rows=1000, n=50001, k=768, out="bf16"),
        # a short text and a small odd vocabulary: many short steps
        dict(name="vocabulary gradient, small", op="vocab_grad", groups=1, rows=37, n=8191, k=256, out="bf16"),
        # 16 workers, each with an output layer of its own
        dict(name="vocabulary gradient, 16 workers", op="vocab_grad", groups=16, rows=2048, n=16384, k=1024, out="bf16"),
        # one model, a long batch
        dict(name="vocabulary gradient, large", op="vocab_grad", groups=1, rows=8192, n=65536, k=2048, out="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["forward", "input_grad", "weight_grad", "act_roundtrip", "act_relu_grad", "act_weight_grad", "vocab_loss",
                     "vocab_grad", "vocab_grad"])
    while True:
        groups, rows = _log(rng, 1, 32), _log(rng, 1, 32768)
        n, k = 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)
        out = rng.choice(["bf16", "f32"])
        if op in ("act_roundtrip", "act_relu_grad"):
            groups, n, k, out = 1, 0, _log(rng, 64, 8192), "bf16"
        elif op.startswith("vocab"):
            groups, rows, n, k, out = _log(rng, 1, 16), _log(rng, 1, 8192), _log(rng, 100, 70000), 8 * _log(rng, 8, 512), "bf16"
            if 6 * rows * n * k > 6.5e12 or groups * n * k > 3e8 or groups * rows * n > 2 ** 31:
                continue
        elif 2 * rows * n * k > 1.0e12 or groups * n * k > 3e8 or groups * rows * max(n, k) > 2 ** 30:
            continue
        return dict(op=op, groups=groups, rows=rows, n=n, k=k, out=out)


def work(case):
    g, m, n, k, op = (case[x] for x in ("groups", "rows", "n", "k", "op"))
    o = 4 if case["out"] == "f32" else 2
    used = min(g, m)                                  # groups without rows need not be read
    if op == "forward":
        return {"bytes": 2 * m * k + 2 * used * n * k + o * m * n, "flops": 2 * m * n * k}
    if op == "input_grad":
        return {"bytes": 2 * m * n + 2 * used * n * k + o * m * k, "flops": 2 * m * n * k}
    if op == "weight_grad":
        return {"bytes": 2 * m * (n + k) + o * g * n * k, "flops": 2 * m * n * k}
    scales = m * -(-k // BLOCK)
    if op == "act_roundtrip":                         # in, out, and the 8-bit form once
        return {"bytes": 5 * m * k + scales, "flops": 0}
    if op == "act_relu_grad":                         # the gate needs the values' signs, not the scales
        return {"bytes": 5 * m * k, "flops": 0}
    if op == "act_weight_grad":
        return {"bytes": 2 * m * n + m * k + scales + o * g * n * k, "flops": 2 * m * n * k}
    if op == "vocab_loss":
        return {"bytes": 2 * m * k + 2 * used * n * k + 8 * m, "flops": 2 * m * n * k}
    return {"bytes": 4 * m * k + 2 * used * n * k + 2 * g * n * k + 8 * m, "flops": 6 * m * n * k}


# ------------------------------------------------------------------------------------------------------- inputs
def _sizes(case, seed):
    """Rows of each group: unequal, the last of four or more groups empty."""
    rng = random.Random("%s %s" % (seed, case["groups"]))
    g, m = case["groups"], case["rows"]
    share = [rng.uniform(0.5, 1.5) for _ in range(g)]
    if g >= 4:
        share[-1] = 0.0
    total, at, offsets = sum(share), 0.0, [0]
    for s in share:
        at += s
        offsets.append(min(m, int(m * at / total + 0.5)))
    offsets[-1] = m
    return offsets


def prepare(case, seed):
    op, g, m, n, k = (case[x] for x in ("op", "groups", "rows", "n", "k"))
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)

    offsets = _sizes(case, seed)
    s = dict(case, offsets=torch.tensor(offsets, dtype=torch.int32, device="cuda"),
             longest=max(b - a for a, b in zip(offsets, offsets[1:])))
    if n:
        # every group's weights lie in a row of a larger matrix: its whole flattened model
        stride = (n * k + k + 63) // 64 * 64
        if op in ("forward", "input_grad") or op.startswith("vocab"):
            scale = (2.0 if op.startswith("vocab") else 1.0) / math.sqrt(k)
            s["w"] = torch.as_strided(normal(g, stride, scale=scale), (g, n, k), (stride, k, 1))
    if op == "forward":
        s["x"] = normal(m, k)
    elif op == "input_grad":
        s["dy"] = normal(m, n, scale=0.01)
    elif op == "weight_grad":
        s["x"], s["dy"] = normal(m, k), normal(m, n, scale=0.01)
    elif op == "act_roundtrip":
        s["x"] = normal(m, k) * torch.exp(torch.randn(m, 1, generator=gen, device="cuda")).to(torch.bfloat16)
    elif op in ("act_relu_grad", "act_weight_grad"):
        act = normal(m, k).clamp(min=0)
        s["q"], s["scales"] = _pack(act)
        s["dy"] = normal(m, n or k, scale=0.01)
    else:
        s["x"] = normal(m, k)
        # frequent and rare tokens, and rows (padding) that take no part
        pick = torch.rand(m, generator=gen, device="cuda")
        label = (torch.exp(pick * math.log(n)) - 1).to(torch.int32).clamp(0, n - 1)
        s["labels"] = torch.where(torch.rand(m, generator=gen, device="cuda") < 0.06, IGNORED, label).to(torch.int32)
    if n and op.endswith("weight_grad") and case["out"] == "f32":
        s["grads"] = torch.as_strided(torch.zeros(g, stride, device="cuda"), (g, n, k), (stride, k, 1))
    if own:
        from paper_1906_12043_b200 import lm
        s["ops"] = lm.LMOps()
        if "q" in s:
            s["packed"] = lm.PackedActivations.from_parts(s["q"], s["scales"])
    return s


# ------------------------------------------------------------------------------------------------------- the operators
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    op, ops = s["op"], s["ops"]
    kind = torch.float32 if s["out"] == "f32" else torch.bfloat16
    if op == "forward":
        return ops.grouped_forward(s["x"], s["w"], s["offsets"], out_dtype=kind)
    if op == "input_grad":
        return ops.grouped_input_grad(s["dy"], s["w"], s["offsets"], out_dtype=kind)
    if op == "weight_grad":
        return ops.grouped_weight_grad(s["dy"], s["x"], s["offsets"], out=s.get("grads"), out_dtype=kind)
    if op == "act_roundtrip":
        return ops.act_unpack(ops.act_pack(s["x"]))
    if op == "act_relu_grad":
        return ops.act_relu_grad(s["dy"], s["packed"])
    if op == "act_weight_grad":
        return ops.grouped_weight_grad(s["dy"], s["packed"], s["offsets"], out=s.get("grads"), out_dtype=kind)
    if op == "vocab_loss":
        return ops.vocab_loss(s["x"], s["w"], s["labels"], s["offsets"])
    return ops.vocab_loss_grad(s["x"], s["w"], s["labels"], s["offsets"])


def _slots(s):
    """For every group and place in it the row that stands there, and whether there is one."""
    at = s["offsets"][:-1, None].long() + torch.arange(s["longest"], device="cuda")
    return at.clamp(max=s["rows"] - 1), at < s["offsets"][1:, None]


def _group_of_rows(s):
    return torch.searchsorted(s["offsets"][1:].long(), torch.arange(s["rows"], device="cuda"), right=True)


def _by_group(x, s):
    at, there = _slots(s)
    return x[at] * there[..., None]


def _by_row(y, s):
    g = _group_of_rows(s)
    return y[g, torch.arange(s["rows"], device="cuda") - s["offsets"][g].long()]


def _power(e):
    """2 to the power e, for whole e from -126 to 127."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _pack(x):
    """8-bit form: whole numbers (rows 16-byte aligned), and for each block of columns and row the power of two that they
    count (its exponent + 127)."""
    m, k = x.shape
    blocks = -(-k // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - k)).view(m, blocks, BLOCK)
    part, e = torch.frexp(v.abs().amax(-1))
    e = torch.where(part == 0, -126, torch.where(part > 127 / 128, e - 6, e - 7)).clamp(min=-126)
    y = v * _power(-e)[..., None]
    q = (torch.sign(y) * y.abs().round().clamp(min=1)).to(torch.int8)
    return q.view(m, -1)[:, :-(-k // 16) * 16].contiguous()[:, :k], (e + 127).to(torch.uint8).t().contiguous()


def _unpack(q, scales):
    unit = _power(scales.t().to(torch.int32) - 127)
    return q.float() * unit.repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _run_plain(s):
    op = s["op"]
    kind = torch.float32 if s["out"] == "f32" else torch.bfloat16
    if op == "forward":
        return _by_row(torch.bmm(_by_group(s["x"].float(), s), s["w"].float().transpose(1, 2)), s).to(kind)
    if op == "input_grad":
        return _by_row(torch.bmm(_by_group(s["dy"].float(), s), s["w"].float()), s).to(kind)
    if op == "weight_grad":
        return torch.bmm(_by_group(s["dy"].float(), s).transpose(1, 2), _by_group(s["x"].float(), s)).to(kind)
    if op == "act_roundtrip":
        return _unpack(*_pack(s["x"])).to(kind)
    if op == "act_relu_grad":
        return torch.where(s["q"] > 0, s["dy"].float(), 0.0).to(kind)
    if op == "act_weight_grad":
        x = _unpack(s["q"], s["scales"])
        return torch.bmm(_by_group(s["dy"].float(), s).transpose(1, 2), _by_group(x, s)).to(kind)
    h, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    logits = _by_row(torch.bmm(_by_group(h, s), w.transpose(1, 2)), s)
    there, label = labels >= 0, labels.clamp(min=0)[:, None]
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    row_loss = torch.where(there, (torch.log(total) + top - logits.gather(1, label))[:, 0], 0.0)
    g = _group_of_rows(s)
    count = _by_group(there.float()[:, None], s).sum((1, 2)).clamp(min=1)
    loss = _by_group(row_loss[:, None], s).sum((1, 2)) / count
    if op == "vocab_loss":
        return loss, row_loss
    dl = e.div_(total).scatter_add(1, label, torch.full_like(total, -1.0)) * (there / count[g])[:, None]
    dl = _by_group(dl, s)
    dh = _by_row(torch.bmm(dl, w), s)
    dw = torch.bmm(dl.transpose(1, 2), _by_group(h, s))
    return loss, row_loss, dh.to(kind), dw.to(kind)


# ------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """From the definitions, group by group, in 64 bits."""
    s = prepare(case, seed)
    op, at = s["op"], s["offsets"].tolist()
    spans = [slice(a, b) for a, b in zip(at, at[1:])]
    wide = {x: s[x].double() for x in ("x", "dy") if x in s}
    if op == "forward":
        return torch.cat([torch.einsum("mk,nk->mn", wide["x"][p], s["w"][g].double()) for g, p in enumerate(spans)])
    if op == "input_grad":
        return torch.cat([torch.einsum("mn,nk->mk", wide["dy"][p], s["w"][g].double()) for g, p in enumerate(spans)])
    if op == "weight_grad":
        return torch.stack([torch.einsum("mn,mk->nk", wide["dy"][p], wide["x"][p]) for p in spans])
    if op == "act_roundtrip":
        got = []
        for part in wide["x"].split(BLOCK, 1):
            most = part.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100).cpu()      # the host's powers of two are exact
            unit = torch.exp2(torch.ceil(torch.log2(most / 127))).cuda()
            got.append(torch.sign(part) * torch.maximum(torch.round(part.abs() / unit), torch.ones_like(part)) * unit)
        return torch.cat(got, 1)
    if op == "act_relu_grad":
        return wide["dy"] * (s["q"] > 0).double()
    if op == "act_weight_grad":
        unit = torch.exp2(s["scales"].double().cpu() - 127).cuda()
        parts = [q.double() * unit[b][:, None] for b, q in enumerate(s["q"].split(BLOCK, 1))]
        x = torch.cat(parts, 1)
        return torch.stack([torch.einsum("mn,mk->nk", wide["dy"][p], x[p]) for p in spans])
    loss, row_loss, dh, dw = [], [], [], []
    for g, p in enumerate(spans):
        h, w, t = wide["x"][p], s["w"][g].double(), s["labels"][p].long()
        use = (t >= 0).nonzero()[:, 0]
        logits = h[use] @ w.T
        logp = logits - torch.logsumexp(logits, 1, keepdim=True)
        here = torch.zeros(h.shape[0], dtype=torch.float64, device="cuda")
        here[use] = -logp[torch.arange(len(use), device="cuda"), t[use]]
        row_loss.append(here)
        loss.append(here.sum() / max(1, len(use)))
        if op == "vocab_grad":
            d = logp.exp_()
            d[torch.arange(len(use), device="cuda"), t[use]] -= 1
            d /= max(1, len(use))
            back = torch.zeros_like(h)
            back[use] = d @ w
            dh.append(back)
            dw.append(d.T @ h[use])
    if op == "vocab_loss":
        return torch.stack(loss), torch.cat(row_loss)
    return torch.stack(loss), torch.cat(row_loss), torch.cat(dh), torch.stack(dw)
