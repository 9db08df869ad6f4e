"""Workloads of a second set of language-model operators: what is measured, on which sizes and inputs.

Three operators, as a worker with a mixture of experts uses them in one training step:

* tokens sorted by expert and back: the sort, the rows in the experts' order, the weighted sum on the way back, and the gradients;
* log probabilities of given tokens, with the entropy and the top alternatives (a router's choice of experts among them), and the
  gradient of the logits;
* an AdamW step over many tensors at once, with the moments in 32 bits or in 8.

``run`` computes them in a plain form (32-bit torch operations, rounded once at the end), or, with ``own`` set, through the package.
"""
import math
import random

import torch

own = False

BLOCK = 128                       # values of 8-bit moments that share a scale
BETAS, EPS, LR, DECAY = (0.9, 0.95), 1e-8, 3e-4, 0.1
STEPS = 20                        # steps an optimizer's state has behind it
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EMPTY = 2.0 ** -100               # a block whose largest value is smaller counts as zero


# ------------------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # a few tokens being generated, two of eight experts each: the calls' own cost is what counts
        dict(name="expert rows, few tokens", op="expert_rows", tokens=17, top=2, groups=8, width=512, type="bf16", absent=False),
        # a training batch: sorted and laid out for the experts' products; some of the tokens are padding
        dict(name="expert rows, batch", op="expert_rows", tokens=16384, top=4, groups=64, width=2048, type="bf16", absent=True),
        # the way back of an odd batch with a width that is no multiple of a power of two
        dict(name="expert join, odd sizes", op="expert_join", tokens=4999, top=6, groups=60, width=1032, type="bf16", absent=False),
        # the gradient of that way back for a large batch: of the experts' results and of the weights
        dict(name="expert join gradient, large", op="expert_join_grad", tokens=16384, top=8, groups=128, width=2048, type="bf16", absent=False),
        # a router: the experts of every token are the top alternatives among 64
        dict(name="router", op="logprobs", rows=16384, vocab=64, top=4, type="f32", given=False, masked=False),
        # four sequences being generated: the sampled tokens' log probabilities and 20 alternatives, odd vocabulary
        dict(name="sampled tokens", op="logprobs", rows=4, vocab=50001, top=20, type="bf16", given=True, masked=True),
        # a batch of answers is scored; five alternatives each
        dict(name="scoring, batch", op="logprobs", rows=4096, vocab=65536, top=5, type="bf16", given=True, masked=False),
        # the logits' gradient from the log probabilities' and the entropy's, a short odd batch
        dict(name="gradient, short", op="logprobs_grad", rows=37, vocab=8191, top=0, type="f32", given=True, masked=False),
        # the same for a training batch
        dict(name="gradient, batch", op="logprobs_grad", rows=4096, vocab=50001, top=0, type="bf16", given=True, masked=True),
        # a small model: the step's own cost is what counts
        dict(name="adamw, small model", op="adamw", tensors=12, values=49_999, bits=32, params="f32", grads="f32", copies=False),
        # the framework's 16 workers of the MLP workload: 6 tensors each, bf16 copies for the products, moments in 8 bits
        dict(name="adamw, 16 workers, 8 bits", op="adamw", tensors=96, values=29_792_416, bits=8, params="f32", grads="f32", copies=True),
        # 16 workers of the ResNet18-sized workload, moments in 32 bits
        dict(name="adamw, large", op="adamw", tensors=992, values=187_032_192, bits=32, params="f32", grads="f32", copies=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["expert_rows", "expert_rows_grad", "expert_join", "expert_join_grad", "logprobs", "logprobs", "logprobs_grad", "logprobs_grad",
                     "adamw", "adamw", "adamw"])
    while True:
        if op.startswith("expert"):
            c = dict(op=op, tokens=_log(rng, 1, 65536), top=_log(rng, 1, 16), groups=_log(rng, 2, 512), width=8 * _log(rng, 8, 1024),
                     type=rng.choice(["bf16", "bf16", "f32"]), absent=rng.random() < 0.3)
            if c["top"] > c["groups"] or c["tokens"] * c["top"] * c["width"] * (2 if c["type"] == "bf16" else 4) > 1.1e9:
                continue
        elif op.startswith("logprobs"):
            c = dict(op=op, rows=_log(rng, 1, 32768), vocab=_log(rng, 8, 160000), top=rng.choice([0, 1, 2, 4, 8, 20, 32]),
                     type=rng.choice(["bf16", "bf16", "f32"]), given=True, masked=rng.random() < 0.3)
            if op == "logprobs":
                c["given"] = rng.random() < 0.7 or c["top"] == 0
            c["top"] = min(c["top"], c["vocab"])
            if c["rows"] * c["vocab"] * (2 if c["type"] == "bf16" else 4) > 5.4e8:
                continue
        else:
            c = dict(op=op, tensors=_log(rng, 1, 1000), values=_log(rng, 1000, 1.5e8), bits=rng.choice([8, 32]), params=rng.choice(["f32", "f32", "bf16"]),
                     grads=rng.choice(["f32", "bf16"]), copies=rng.random() < 0.4)
            c["copies"] = c["copies"] and c["params"] == "f32"
            if c["values"] < 8 * c["tensors"]:
                continue
        return c


def work(case):
    op = case["op"]
    size = 2 if case.get("type") == "bf16" else 4
    if op.startswith("expert"):
        t, n, d = case["tokens"], case["tokens"] * case["top"], case["width"] * size
        if op == "expert_rows":                                  # the experts' numbers, the tokens; the order and the places, the rows
            return {"bytes": 4 * n + t * d + 8 * n + 8 * case["groups"] + n * d, "flops": 0}
        if op == "expert_rows_grad":
            return {"bytes": 4 * n + n * d + t * d, "flops": n * case["width"]}
        if op == "expert_join":
            return {"bytes": 8 * n + n * d + t * d, "flops": 2 * n * case["width"]}
        return {"bytes": 12 * n + t * d + 2 * n * d, "flops": 3 * n * case["width"]}
    if op.startswith("logprobs"):
        m, values = case["rows"], case["rows"] * case["vocab"]
        if op == "logprobs":
            return {"bytes": values * size + m * (8 + (8 if case["given"] else 0) + 8 * case["top"]), "flops": 5 * values}
        return {"bytes": 2 * values * size + m * (20 + 8 * case["top"]), "flops": 5 * values}
    p, g = (2 if case[x] == "bf16" else 4 for x in ("params", "grads"))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 8     # 8 bits: the moments are read out as well
    return {"bytes": case["values"] * (2 * p + g + state + (2 if case["copies"] else 0)), "flops": 16 * case["values"]}


# ------------------------------------------------------------------------------------------------------- inputs
def _starts(case):
    """Where each tensor lies in a flat buffer, [(start, values)], and the buffer's size: half of the tensors are vectors, the
    others matrices of unequal size; each starts at a multiple of 128 values."""
    n, left = case["tensors"], case["values"]
    share = [(1 if i % 2 else 300) * (1 + (i * 37) % 11) for i in range(n)]
    total, at, found = sum(share), 0, []
    for i, s in enumerate(share):
        size = max(1, case["values"] * s // total) if i < n - 1 else max(1, left)
        left -= size
        found.append((at, size))
        at += -(-size // BLOCK) * BLOCK
    return found, at


def _values(flat, starts):
    return [flat[a:a + n] for a, n in starts]


def prepare(case, seed):
    op = case["op"]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, type="f32"):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(TYPES[type])

    s = dict(case)
    if op.startswith("expert"):
        t, k, e, d = (case[x] for x in ("tokens", "top", "groups", "width"))
        # some experts are chosen more often than others, never twice for one token
        liked = torch.randn(e, generator=gen, device="cuda")
        chosen = (torch.rand(t, e, generator=gen, device="cuda").log_().neg_().log_().neg_() + liked).topk(k, 1).indices.to(torch.int32)
        if case["absent"]:                                       # padding: tokens that no expert sees
            chosen[torch.rand(t, generator=gen, device="cuda") < 0.1] = -1
        s["experts"] = chosen
        s["weights"] = torch.softmax(normal(t, k), 1)
        if op == "expert_rows":
            s["x"] = normal(t, d, type=case["type"])
        else:
            s["rows"] = normal(t * k, d, type=case["type"])
            if op == "expert_join_grad":
                s["dy"] = normal(t, d, scale=0.01, type=case["type"])
            s["place"] = _sort(chosen, e)[3]
    elif op.startswith("logprobs"):
        m, v = case["rows"], case["vocab"]
        s["logits"] = normal(m, v, scale=2.0, type=case["type"])
        if case["masked"]:                                       # entries that may not be chosen, among them what fills the vocabulary up
            s["logits"][:, v - v // 50:] = float("-inf")
        s["tokens"] = None
        if case["given"]:
            pick = torch.rand(m, generator=gen, device="cuda")
            s["tokens"] = (torch.exp(pick * math.log(v - v // 50)) - 1).to(torch.int32).clamp(0, v - v // 50 - 1)
            if m > 8:                                            # rows of a prompt or of padding take no part
                s["tokens"][torch.rand(m, generator=gen, device="cuda") < 0.06] = -1
        if op == "logprobs_grad":
            s["known"] = _logprobs(s["logits"], s["tokens"], case["top"])
            s["d_logp"], s["d_entropy"] = normal(m, scale=0.01), normal(m, scale=0.001)
            s["d_top"] = normal(m, case["top"], scale=0.01) if case["top"] else None
    else:
        starts, size = _starts(case)
        s["starts"], s["at"] = starts, STEPS
        inside = torch.zeros(size, device="cuda")
        for x in _values(inside, starts):
            x.fill_(1.0)
        p = normal(size, scale=0.05) * inside
        s["p"] = p.to(TYPES[case["params"]])
        s["copy"] = p.bfloat16() if case["copies"] else None
        width = torch.exp(normal(size))                          # gradients of unequal size
        s["g"] = (normal(size, scale=0.01) * width * inside).to(TYPES[case["grads"]])
        s["m"] = normal(size, scale=0.003) * width * inside
        s["v"] = (normal(size, scale=0.01) * width * inside) ** 2
        s["decay"] = torch.zeros(size, device="cuda")            # the matrices' weights decay, the vectors' do not
        for x in _values(s["decay"], starts[::2]):
            x.fill_(DECAY)
        if case["bits"] == 8 and not own:
            s["m"], s["v"] = _codes(s["m"], s["v"].sqrt())
    if own:
        from paper_1906_12043_b200 import lm, optim
        if op == "adamw":
            s["grad_list"] = _values(s["g"], starts)
            s["opt"] = optim.AdamW(_values(s["p"], starts), lr=LR, betas=BETAS, eps=EPS, weight_decay=[DECAY if i % 2 == 0 else 0.0 for i in range(len(starts))],
                                   state_bits=case["bits"], copies=_values(s["copy"], starts) if case["copies"] else None)
            s["opt"].load_moments(STEPS, s.pop("m"), s.pop("v"))
            s.pop("decay")
        else:
            s["ops"] = lm.LMOps()
            if op.startswith("expert") and op != "expert_rows":
                s["plan"] = s["ops"].expert_sort(s["experts"], case["groups"])
            if op == "logprobs_grad":
                k = s["known"]
                s["known"] = lm.TokenLogprobs(k[0], k[1], k[2], *(k[3:] if case["top"] else (None, None)))
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _sort(experts, groups):
    """offsets, counts, order, place: slots that take no part lie behind the last expert's, and count as its rows in the offsets."""
    flat = experts.reshape(-1)
    there = flat >= 0
    order = torch.sort(torch.where(there, flat, groups), stable=True).indices
    row = torch.empty_like(order)
    row[order] = torch.arange(order.numel(), device="cuda")
    counts = (flat[None, :] == torch.arange(groups, device="cuda")[:, None]).sum(1) if flat.numel() * groups < 2 ** 22 else \
        torch.zeros(groups, dtype=torch.int64, device="cuda").scatter_add_(0, flat.clamp(min=0).long(), there.long())
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    offsets[-1] = flat.numel()
    place = torch.where(there, row, -1 - row).view(experts.shape)
    return tuple(x.to(torch.int32) for x in (offsets, counts, order, place))


def _key(x):
    """Whole numbers in the order of the values (equal values, equal numbers)."""
    b = (x.float() + 0.0).view(torch.int32)
    return torch.where(b < 0, b ^ 0x7FFFFFFF, b).long()


def _logprobs(logits, tokens, top):
    x = logits.float()
    most = x.amax(1, keepdim=True)
    most = torch.where(most > -math.inf, most, 0.0)
    e = torch.exp(x - most)
    total = e.sum(1)
    z = torch.log(total)
    entropy = torch.where(total > 0, z - torch.where(e > 0, e * (x - most), 0.0).sum(1) / total, 0.0)
    z = z + most[:, 0]
    there = torch.ones_like(z, dtype=torch.bool) if tokens is None else tokens >= 0
    empty = z == -math.inf
    known = [None if tokens is None else
             torch.where(there, torch.where(empty, z, x.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0] - z), 0.0)]
    known += [torch.where(there, entropy, 0.0), torch.where(there, z, 0.0)]
    if top:
        v = x.shape[1]
        best = v - 1 - ((_key(x) << 32) + torch.arange(v - 1, -1, -1, device="cuda")).topk(top, 1).values % 2 ** 32
        logp = torch.where(empty[:, None], z[:, None], x.gather(1, best) - z[:, None])
        known += [torch.where(there[:, None], logp, 0.0), torch.where(there[:, None], best, -1).to(torch.int32)]
    return known


def _codes(m, r):
    """The moments in 8 bits: whole numbers and their units, blocks of 128.  r: the second moments' roots."""
    m, r = m.view(-1, BLOCK), r.view(-1, BLOCK)
    am, ar = m.abs().amax(1, keepdim=True), r.amax(1, keepdim=True)
    zero = torch.zeros_like(am)
    um, ur = torch.where(am >= EMPTY, am * (1 / 16129), zero), torch.where(ar >= EMPTY, ar * (1 / 65025), zero)
    im, ir = torch.where(am >= EMPTY, torch.full_like(am, 16129) / am, zero), torch.where(ar >= EMPTY, torch.full_like(ar, 65025) / ar, zero)
    c = torch.round(torch.sqrt(m.abs() * im)) * torch.sign(m)
    d = torch.round(torch.sqrt(r * ir))
    d = torch.where((r > 0) & (ir > 0), d.clamp(min=1), d)
    return (c.to(torch.int8), um), (d.to(torch.uint8), ur)


def _moments(m, v):
    c, d = m[0].float(), v[0].float()
    r = (d * d) * v[1]
    return ((c * c.abs()) * m[1]).view(-1), (r * r).view(-1)


def _adamw(s):
    s["at"] += 1
    eight = s["bits"] == 8
    m, v = _moments(s["m"], s["v"]) if eight else (s["m"], s["v"])
    g = s["g"].float()
    b1, b2 = BETAS
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    r = torch.sqrt(v)
    c1, c2 = 1 / (1 - b1 ** s["at"]), 1 / math.sqrt(1 - b2 ** s["at"])
    p = s["p"].float()
    p = p * (1 - LR * s["decay"]) - (LR * c1) * m / (r * c2 + EPS)
    s["p"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if eight:
        s["m"], s["v"] = _codes(m, r)
        return _moments(s["m"], s["v"])
    s["m"].copy_(m)
    s["v"].copy_(v)
    return s["m"], s["v"]


def _run_own(s):
    op = s["op"]
    if op == "adamw":
        s["opt"].step(s["grad_list"])
        return [s["p"], *s["opt"].moments()] + ([s["copy"]] if s["copies"] else [])
    ops = s["ops"]
    if op == "expert_rows":
        plan = ops.expert_sort(s["experts"], s["groups"])
        return [plan.offsets, plan.counts, plan.order, plan.place, ops.expert_rows(s["x"], plan)]
    if op == "expert_rows_grad":
        return ops.expert_rows_grad(s["rows"], s["plan"])
    if op == "expert_join":
        return ops.expert_join(s["rows"], s["plan"], s["weights"])
    if op == "expert_join_grad":
        return ops.expert_join_grad(s["dy"], s["rows"], s["plan"], s["weights"])
    if op == "logprobs":
        return [x for x in ops.token_logprobs(s["logits"], s["tokens"], top=s["top"]) if x is not None]
    return ops.token_logprobs_grad(s["logits"], s["tokens"], s["known"], s["d_logp"], s["d_entropy"], s["d_top"])


def run(s):
    if own:
        return _run_own(s)
    op = s["op"]
    if op == "adamw":
        return [s["p"], *_adamw(s)] + ([s["copy"]] if s["copies"] else [])
    if op == "expert_rows":
        offsets, counts, order, place = _sort(s["experts"], s["groups"])
        rows = s["x"][order.long() // s["top"]]
        if s["absent"]:
            rows = torch.where((s["experts"].reshape(-1)[order.long()] >= 0)[:, None], rows, 0.0)
        return [offsets, counts, order, place, rows]
    if op.startswith("expert"):
        there, at = (s["place"] >= 0)[:, :, None], torch.where(s["place"] >= 0, s["place"], -1 - s["place"]).long()
        rows = s["rows"].float()[at]
        if op == "expert_rows_grad":
            return torch.where(there, rows, 0.0).sum(1).to(s["rows"].dtype)
        if op == "expert_join":
            return torch.where(there, rows * s["weights"][:, :, None], 0.0).sum(1).to(s["rows"].dtype)
        dy = s["dy"].float()[:, None, :]
        back = torch.empty_like(s["rows"])
        back[at.view(-1)] = torch.where(there, dy * s["weights"][:, :, None], 0.0).to(back.dtype).view(-1, back.shape[1])
        return back, torch.where(there, dy * rows, 0.0).sum(2)
    if op == "logprobs":
        return [x for x in _logprobs(s["logits"], s["tokens"], s["top"]) if x is not None]
    logp, entropy, z = (x[:, None] for x in s["known"][:3])
    there, t = (s["tokens"] >= 0)[:, None], s["tokens"].clamp(min=0).long()[:, None]
    own_logp = s["logits"].float() - z
    p = torch.exp(own_logp)
    every = s["d_logp"][:, None] if s["d_top"] is None else s["d_logp"][:, None] + s["d_top"].sum(1, keepdim=True)
    d = torch.where(p > 0, -p * (every + s["d_entropy"][:, None] * (own_logp + entropy)), 0.0)
    d.scatter_add_(1, t, s["d_logp"][:, None])
    if s["d_top"] is not None:
        d.scatter_add_(1, s["known"][4].clamp(min=0).long(), s["d_top"])
    return torch.where(there, d, 0.0).to(s["logits"].dtype)


# ------------------------------------------------------------------------------------------------------- in 64 bits
def _f32(x):
    return x.float().double()


def _exact_adamw(case, s):
    """32 bits: the formulas.  8 bits: the definition names the roundings to fp32 between the old state and the new one."""
    b1, b2 = BETAS
    m, v, g, p = s["m"].double(), s["v"].double(), s["g"].double(), s["p"].double()
    t = STEPS + 1
    if case["bits"] == 8:
        def coded(m, r):
            found = []
            for x, top, least in ((m, 127, 0), (r, 255, 1)):
                x = x.view(-1, BLOCK)
                most = x.abs().amax(1, keepdim=True)
                unit, per = _f32(most * _f32(torch.full_like(most, 1 / top ** 2))), _f32(top ** 2 / most.clamp(min=EMPTY))
                c = torch.floor(_f32(torch.sqrt(_f32(x.abs() * per))) + 0.5)
                half = _f32(torch.sqrt(_f32(x.abs() * per))) % 1 == 0.5               # ties go to the even one
                c = torch.where(half & (c % 2 == 1), c - 1, c)
                c = torch.where(x != 0, c.clamp(min=least), 0 * c)
                found.append(torch.where(most >= EMPTY, c * c * x.sign() * unit, 0 * c).view(-1))
            return _f32(found[0]), _f32(_f32(found[1]) ** 2)
        m, v = coded(m, _f32(torch.sqrt(v)))
        w = [_f32(torch.tensor(x, dtype=torch.float64, device="cuda")) for x in (b1, 1 - b1, b2, 1 - b2)]
        m = _f32(_f32(m * w[0]) + _f32(g * w[1]))
        v = _f32(_f32(v * w[2]) + _f32(_f32(g * g) * w[3]))
        r = _f32(torch.sqrt(v))
        kept = coded(m, r)
    else:
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        r, kept = v.sqrt(), (m, v)
    p = p - LR * s["decay"].double() * p - LR * (m / (1 - b1 ** t)) / (r / math.sqrt(1 - b2 ** t) + EPS)
    return [p, *kept] + ([p] if case["copies"] else [])


def exact(case, seed):
    """From the definitions, in 64 bits, a stretch of rows at a time."""
    op = case["op"]
    if op == "adamw":                                     # (the state before its coding, which is written above once more)
        return _exact_adamw(case, prepare(dict(case, bits=32), seed))
    s = prepare(case, seed)
    if op.startswith("expert"):
        e, k = s["experts"].cpu().reshape(-1).tolist(), case["top"]
        lists = [[] for _ in range(case["groups"] + 1)]
        for slot, x in enumerate(e):
            lists[x if x >= 0 else case["groups"]].append(slot)
        order = torch.tensor([slot for x in lists for slot in x], device="cuda")
        live = len(e) - len(lists[-1])
        if op == "expert_rows":
            ends = torch.tensor([0] + [len(x) for x in lists[:-1]], device="cuda").cumsum(0)
            ends[-1] = len(e)
            place = torch.empty(len(e), dtype=torch.int64, device="cuda")
            at = torch.arange(len(e), device="cuda")
            place[order] = torch.where(at < live, at, -1 - at)
            rows = s["x"].double()[torch.div(order, k, rounding_mode="floor")]
            rows[live:] = 0
            return [ends, torch.tensor([len(x) for x in lists[:-1]], device="cuda"), order, place.view(case["tokens"], k), rows]
        token = torch.div(order, k, rounding_mode="floor")[:live]
        rows, w = s["rows"][:live], s["weights"].double().view(-1)[order[:live]][:, None]
        wide = lambda x: x.double()  # noqa: E731
        if op in ("expert_join", "expert_rows_grad"):
            y = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device="cuda")
            return y.index_add_(0, token, wide(rows) * w if op == "expert_join" else wide(rows))
        dy = s["dy"].double()[token]
        dw = torch.zeros(len(e), dtype=torch.float64, device="cuda")
        dw[order[:live]] = torch.einsum("nd,nd->n", dy, wide(rows))
        back = torch.zeros(len(e), case["width"], dtype=torch.float64, device="cuda")
        back[:live] = dy * w
        return back, dw.view(case["tokens"], k)
    found = []
    step = max(1, 2 ** 26 // case["vocab"])
    for a in range(0, case["rows"], step):
        x = s["logits"][a:a + step].double()
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        h = -torch.where(p > 0, p * lp, 0.0).sum(1)
        t = None if s["tokens"] is None else s["tokens"][a:a + step].long()
        there = torch.ones(len(x), dtype=torch.bool, device="cuda") if t is None else t >= 0
        row = torch.arange(len(x), device="cuda")
        if op == "logprobs":
            part = [] if t is None else [lp[row, t.clamp(min=0)]]
            part += [h, torch.logsumexp(x, 1)]
            if case["top"]:
                best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
                part += [lp.gather(1, best), best]
            found.append([torch.where(there if y.dim() == 1 else there[:, None], y, -1 if y.dtype == torch.int64 else 0.0) for y in part])
        else:
            d = torch.zeros_like(x)
            d[row, t.clamp(min=0)] += s["d_logp"][a:a + step].double()
            if case["top"]:
                best = s["known"][4][a:a + step].clamp(min=0).long()
                d.scatter_add_(1, best, s["d_top"][a:a + step].double())
            d -= p * d.sum(1, keepdim=True)
            d -= s["d_entropy"][a:a + step].double()[:, None] * torch.where(p > 0, p * (lp + h[:, None]), 0.0)
            found.append([torch.where(there[:, None], d, 0.0)])
    joined = [torch.cat(x) for x in zip(*found)]
    return joined if op == "logprobs" else joined[0]
