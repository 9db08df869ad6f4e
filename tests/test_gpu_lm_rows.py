"""Tokens sorted by expert and back, and log probabilities of tokens (lm.LMOps), against plain implementations in 64 bits.

Tolerances, derived before the first run:

* the sort, the rows and the order of the alternatives are exact.
* a sum of k products in fp32, rounded once each: k * 2^-24 * (sum of magnitudes), plus half a step of a bf16 result (2^-8, fp32 2^-24 of the value).
* a dot product of D products: a thread adds at most D / 32 + 8 of them one after the other, then 5 + 3 joins: (D / 32 + 16) * 2^-24 * (sum of magnitudes).
* log probabilities: t = (l - m) * scale * log2 e carries three roundings (2^-24 each, relative to |t|) and the exponential 2^-22, so that a term of the sum is off by
  at most 2^-22 + 3 * 2^-24 * |t|, and terms of |t| > 24 are below 2^-24 of the sum: 2^-22 + 72 * 2^-24 = 19 * 2^-22 for each that counts.  The sums add at most
  V / 128 + 64 terms one after the other.  With s = 19 * 2^-22 + (V / 128 + 64) * 2^-24, ln S1 is off by s, Z and log p by s + 2^-22 * (1 + |y| + |Z|), and the entropy by
  s * (2 + ln V) (S2 / S1 is at most ln V, and each of its terms is off by at most s of itself).
* the gradient: log p is off by a = 2^-22 * (1 + |y| + |Z|) + (the given log_sum's own error, none: the test gives it in fp32, 2^-24 |Z|), p by 2^-22 + a relative, so that a
  term p * (A + g (log p + H)) is off by p * ((2^-21 + a) * (|A| + |g| |log p + H|) + |g| (a + 2^-23 H)), plus the result's rounding.  ex2.approx flushes results below 2^-126 to zero.
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def lm():
    from paper_1906_12043_b200 import build, lm
    build.build()
    return lm


@pytest.fixture(scope="module")
def ops(lm):
    o = lm.LMOps()
    yield o
    o.check()
    o.destroy()


def half_step(t):
    return torch.finfo(t).eps / 2


def gaussian(seed, *shape, scale=1.0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def choices(seed, T, k, E, absent=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    e = torch.randint(0, E, (T, k), generator=g, device="cuda", dtype=torch.int32)
    if absent:
        e[torch.rand(T, k, generator=g, device="cuda") < absent] = -1
    return e


# ------------------------------------------------------------------------------------------------------- experts
def plain_sort(experts, E):
    flat = experts.reshape(-1).cpu().tolist()
    rows = [[] for _ in range(E + 1)]
    for s, e in enumerate(flat):
        rows[e if 0 <= e < E else E].append(s)
    order = [s for r in rows for s in r]
    live = len(flat) - len(rows[E])
    place = [0] * len(flat)
    for r, s in enumerate(order):
        place[s] = r if r < live else ~r
    offsets = [0]
    for r in rows[:-1]:
        offsets.append(offsets[-1] + len(r))
    offsets[-1] = len(flat)
    return offsets, [len(r) for r in rows[:-1]], order, place


SORTS = [(0, 2, 4), (1, 1, 1), (1, 8, 8), (3, 5, 7), (37, 2, 8), (1000, 1, 1000), (1024, 4, 64), (1025, 4, 1024), (1366, 3, 5), (4097, 1, 3), (9999, 7, 60), (40000, 8, 128),
         (7000, 32, 1023)]


@pytest.mark.parametrize("T,k,E", SORTS)
@pytest.mark.parametrize("absent", [0.0, 0.3, 1.0])
def test_slots_in_the_order_of_their_experts(ops, T, k, E, absent):
    e = choices(T + k, T, k, E, absent)
    plan = ops.expert_sort(e, E)
    offsets, counts, order, place = plain_sort(e, E)
    assert plan.offsets.tolist() == offsets and plan.counts.tolist() == counts
    assert plan.order.tolist() == order and plan.place.reshape(-1).tolist() == place
    assert plan.place.shape == (T, k)
    ops.check()


def test_one_expert_takes_all_and_views_of_choices(ops):
    for T, k in ((5000, 4), (100, 2)):
        wide = torch.full((T, k + 3), 5, dtype=torch.int32, device="cuda")
        plan = ops.expert_sort(wide[:, 1:1 + k], 9)
        assert plan.order.tolist() == list(range(T * k)) and plan.offsets.tolist() == [0] * 6 + [T * k] * 4
        wide[:, 1:1 + k] = choices(1, T, k, 9)
        got, want = ops.expert_sort(wide[:, 1:1 + k], 9), ops.expert_sort(wide[:, 1:1 + k].contiguous(), 9)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("T,k,E", [(33, 2, 8), (3000, 4, 16)])
def test_a_number_beyond_the_experts_takes_no_part_and_is_reported(ops, lm, T, k, E):
    from paper_1906_12043_b200.engine import CocodError
    e = choices(2, T, k, E)
    bad = e.clone()
    bad[T // 2, 0] = E
    plan = ops.expert_sort(bad, E)
    with pytest.raises(CocodError):
        ops.check()
    ops.check()
    offsets, counts, order, place = plain_sort(bad, E)
    assert plan.offsets.tolist() == offsets and plan.counts.tolist() == counts and plan.order.tolist() == order and plan.place.reshape(-1).tolist() == place


ROWS = [(1, 1, 1, 8), (5, 3, 4, 7), (17, 2, 8, 512), (100, 8, 16, 264), (64, 1, 2, 1), (333, 6, 60, 1032), (50, 32, 40, 96), (9, 2, 5, 9000), (700, 4, 9, 2047)]


@pytest.mark.parametrize("T,k,E,D", ROWS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("absent", [0.0, 0.25])
def test_there_and_back(ops, T, k, E, D, dtype, absent):
    plan = ops.expert_sort(choices(T, T, k, E, absent), E)
    there = plan.place >= 0
    at = torch.where(there, plan.place, ~plan.place).long()
    x, ys, dy = gaussian(1, T, D, dtype=dtype), gaussian(2, T * k, D, dtype=dtype), gaussian(3, T, D, dtype=dtype)
    w = gaussian(4, T, k)
    if not there.all():
        ys[at[~there]] = float("nan")                       # what such rows hold is not looked at
    rows = ops.expert_rows(x, plan)
    want = torch.zeros_like(rows)
    want[at[there]] = x[:, None].expand(T, k, D)[there]
    assert torch.equal(rows, want)
    wide = torch.where(there[..., None], ys.double()[at], 0.0)
    for out_dtype in (torch.bfloat16, torch.float32):
        for weights in (w, None):
            got = ops.expert_rows_grad(ys, plan, out_dtype=out_dtype) if weights is None else ops.expert_join(ys, plan, w, out_dtype=out_dtype)
            f = (torch.ones_like(w) if weights is None else w).double()[..., None]
            y, size = (f * wide).sum(1), (f * wide).abs().sum(1)
            assert got.dtype == out_dtype
            assert ((got.double() - y).abs() <= half_step(out_dtype) * y.abs() + 1.01 * (k + 1) * 2.0 ** -24 * size).all()
    drows, dw = ops.expert_join_grad(dy, ys, plan, w)
    back = torch.zeros(T * k, D, dtype=torch.float64, device="cuda")
    back[at[there]] = (w.double()[..., None] * dy.double()[:, None])[there]
    # (a product of fp32 is rounded to fp32, then to the result's type)
    assert ((drows.double() - back).abs() <= 1.01 * (half_step(dtype) + 2.0 ** -24) * back.abs()).all()
    assert (drows[at[~there]] == 0).all()
    products = wide * dy.double()[:, None]
    assert ((dw.double() - products.sum(2)).abs() <= (D / 32 + 16) * 2.0 ** -24 * products.abs().sum(2)).all()
    assert (dw[~there] == 0).all()
    ops.check()


def test_gradients_are_the_formulas(ops):
    """Against autograd in 64 bits through the same gather and weighted sum."""
    T, k, E, D = 40, 3, 6, 72
    e = choices(9, T, k, E, 0.2)
    plan = ops.expert_sort(e, E)
    at, there = torch.where(plan.place >= 0, plan.place, ~plan.place).long(), plan.place >= 0
    x, w, dy, mix = gaussian(1, T, D), gaussian(2, T, k), gaussian(3, T, D), gaussian(4, T * k, D)
    xd, wd = x.double().requires_grad_(True), w.double().requires_grad_(True)
    rows = torch.zeros(T * k, D, dtype=torch.float64, device="cuda").index_put((at[there],), xd[:, None].expand(T, k, D)[there])
    hidden = rows * mix.double()
    y = (torch.where(there[..., None], hidden[at], 0.0) * wd[..., None]).sum(1)
    y.backward(dy.double())
    h = ops.expert_rows(x, plan) * mix
    dh, dw = ops.expert_join_grad(dy, h, plan, w)
    dx = ops.expert_rows_grad(dh * mix, plan)
    assert ((dx.double() - xd.grad).abs() <= 16 * 2.0 ** -24 * (xd.grad.abs() + 8)).all()
    assert ((dw.double() - wd.grad).abs() <= 64 * 2.0 ** -24 * 64).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lead", [0, 1, 8])
def test_views_and_their_surroundings(ops, dtype, lead):
    """Rows of a larger matrix, at any alignment; nothing beside them is written."""
    T, k, E, D = 90, 3, 7, 136
    plan = ops.expert_sort(choices(5, T, k, E, 0.1), E)
    w = gaussian(4, T, k)

    def inside(t):
        whole = torch.full((t.shape[0] + 2, t.shape[1] + 24), 7.0, dtype=t.dtype, device="cuda")
        view = whole[1:-1, lead:lead + t.shape[1]]
        view.copy_(t)
        return view, whole

    def untouched(view, whole):
        w2 = whole.clone()
        w2[1:-1, lead:lead + view.shape[1]] = 7
        return (w2 == 7).all()

    x, ys, dy = gaussian(1, T, D, dtype=dtype), gaussian(2, T * k, D, dtype=dtype), gaussian(3, T, D, dtype=dtype)
    out, whole = inside(torch.zeros(T * k, D, dtype=dtype, device="cuda"))
    assert ops.expert_rows(inside(x)[0], plan, out=out) is out
    assert torch.equal(out, ops.expert_rows(x, plan)) and untouched(out, whole)
    y, whole = inside(torch.zeros(T, D, dtype=dtype, device="cuda"))
    ops.expert_join(inside(ys)[0], plan, w, out=y)
    assert torch.equal(y, ops.expert_join(ys, plan, w)) and untouched(y, whole)
    d, whole = inside(torch.zeros(T * k, D, dtype=dtype, device="cuda"))
    _, dw = ops.expert_join_grad(inside(dy)[0], inside(ys)[0], plan, w, out=d)
    want, dw2 = ops.expert_join_grad(dy, ys, plan, w)
    assert torch.equal(d, want) and untouched(d, whole)
    products = ys.double().abs()[torch.where(plan.place >= 0, plan.place, ~plan.place).long()] * dy.double().abs()[:, None]
    assert ((dw - dw2).abs().double() <= 2 * (D + 16) * 2.0 ** -24 * products.sum(2)).all()


def at_the_end(t):
    """The same values where a segment of the allocator's memory ends: a read behind them leaves mapped memory."""
    size = max(32 << 20, -(-t.numel() * t.element_size() // (2 << 20)) * (2 << 20))
    whole = torch.empty(size, dtype=torch.uint8, device="cuda")
    bytes_ = t.numel() * t.element_size()
    view = whole[size - bytes_:].view(t.dtype).view(t.shape)
    view.copy_(t)
    return view


@pytest.mark.parametrize("T,k,D", [(1, 1, 1), (76, 8, 3), (33, 1, 5), (40, 2, 33), (20, 4, 130), (9, 3, 264), (5, 2, 2056), (7, 6, 1031)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_operands_that_end_where_memory_ends(ops, T, k, D, dtype):
    """Read-only loads of bf16 are assembly that the compiler may move before the condition they stand behind: lanes without a piece read behind the
    last row (seen as an illegal address once in thousands of calls, where the operand lay at the end of mapped memory)."""
    torch.cuda.empty_cache()
    plan = ops.expert_sort(at_the_end(choices(1, T, k, 4, 0.2)), 4)
    plan = plan._replace(place=at_the_end(plan.place))
    x, ys, dy, w = (at_the_end(t) for t in (gaussian(1, T, D, dtype=dtype), gaussian(2, T * k, D, dtype=dtype), gaussian(3, T, D, dtype=dtype), gaussian(4, T, k)))
    own = [t.clone() for t in (x, ys, dy, w)]
    assert torch.equal(ops.expert_rows(x, plan), ops.expert_rows(own[0], plan))
    assert torch.equal(ops.expert_join(ys, plan, w), ops.expert_join(own[1], plan, own[3]))
    assert torch.equal(ops.expert_rows_grad(ys, plan), ops.expert_rows_grad(own[1], plan))
    got, want = ops.expert_join_grad(dy, ys, plan, w, out=at_the_end(torch.zeros_like(ys))), ops.expert_join_grad(own[2], own[1], plan, own[3])
    assert torch.equal(got[0], want[0])
    products = (own[2].double().abs()[:, None] * own[1].double().abs()[torch.where(plan.place >= 0, plan.place, ~plan.place).long()]).sum(2)
    assert ((got[1] - want[1]).abs().double() <= 2 * (D + 16) * 2.0 ** -24 * products).all()
    for V in (D, 70 * D):
        logits = at_the_end(gaussian(5, T, V, dtype=dtype))
        top = min(V, 5)
        a, b = ops.token_logprobs(logits, top=top), ops.token_logprobs(logits.clone(), top=top)
        assert torch.equal(a.top_tokens, b.top_tokens)
        g = gaussian(6, T)
        ops.token_logprobs_grad(logits, None, a, d_entropy=g, out=logits)
        assert torch.isfinite(logits).all()
    ops.check()


def test_a_place_beyond_the_rows_is_left_out_and_reported(ops, lm):
    from paper_1906_12043_b200.engine import CocodError
    T, k, E, D = 20, 2, 4, 64
    plan = ops.expert_sort(choices(5, T, k, E), E)
    x, ys = gaussian(1, T, D, dtype=torch.bfloat16), gaussian(2, T * k, D, dtype=torch.bfloat16)
    for bad_row in (T * k, 2 ** 31 - 1, -1 - T * k, -2 ** 31):
        place = plan.place.clone()
        place[3, 1] = bad_row
        bad = plan._replace(place=place)
        out = torch.full((T * k, D), 7.0, dtype=torch.bfloat16, device="cuda")
        ops.expert_rows(x, bad, out=out)
        want = ops.expert_rows(x, plan)
        want[plan.place[3, 1].long()] = 7
        assert torch.equal(out, want)
        with pytest.raises(CocodError):
            ops.check()
        y = ops.expert_rows_grad(ys, bad, out_dtype=torch.float32)
        assert torch.equal(y[3], ys[plan.place[3, 0].long()].float())
        with pytest.raises(CocodError):
            ops.check()


def test_more_than_2_to_the_31_values(ops):
    T, k, E, D = 70000, 4, 8, 8192                              # 2.3e9 values of rows
    plan = ops.expert_sort(choices(6, T, k, E), E)
    x = gaussian(1, T, 64, dtype=torch.bfloat16).repeat(1, D // 64)
    rows = ops.expert_rows(x, plan)
    token = plan.order.long() // k
    for a in range(0, T * k, 20000):
        assert torch.equal(rows[a:a + 20000], x[token[a:a + 20000]])
    y = ops.expert_rows_grad(rows, plan)
    assert torch.equal(y, x * 4)
    ops.check()


def test_refusals(ops, lm):
    T, k, E, D = 8, 2, 4, 16
    e = choices(1, T, k, E)
    plan = ops.expert_sort(e, E)
    x, ys, w = gaussian(1, T, D), gaussian(2, T * k, D), gaussian(3, T, k)
    for bad in (e.long(), e.cpu(), e.t(), e[0], torch.zeros(T, 33, dtype=torch.int32, device="cuda"), torch.zeros(T, 0, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            ops.expert_sort(bad, E)
    for bad in (0, -1, 1025):
        with pytest.raises(ValueError):
            ops.expert_sort(e, bad)
    for call in (lambda: ops.expert_rows(x[:-1], plan), lambda: ops.expert_rows(x.half(), plan), lambda: ops.expert_rows(x.t(), plan),
                 lambda: ops.expert_rows(x, plan, out=ys[:-1]), lambda: ops.expert_rows(x, plan, out=ys.bfloat16()), lambda: ops.expert_rows(x.cpu(), plan),
                 lambda: ops.expert_join(ys, plan, w.double()), lambda: ops.expert_join(ys, plan, w[:, :1]), lambda: ops.expert_join(ys, plan, None),
                 lambda: ops.expert_join(ys[1:], plan, w), lambda: ops.expert_join(ys, plan, w, out=ys[:T]), lambda: ops.expert_join(ys, plan, w, out_dtype=torch.float16),
                 lambda: ops.expert_join_grad(x, ys, plan, w, out=ys), lambda: ops.expert_join_grad(x.bfloat16(), ys, plan, w),
                 lambda: ops.expert_join_grad(x, ys, plan, w.t()), lambda: ops.expert_rows(x, plan._replace(place=plan.place.long())),
                 lambda: ops.token_logprobs(ys, top=33), lambda: ops.token_logprobs(ys, top=17), lambda: ops.token_logprobs(ys, top=-1), lambda: ops.token_logprobs(ys.half()),
                 lambda: ops.token_logprobs(ys, plan.order.long()), lambda: ops.token_logprobs(ys, plan.order[1:]), lambda: ops.token_logprobs(ys.t())):
        with pytest.raises(ValueError):
            call()
    from paper_1906_12043_b200.engine import CocodError
    for bad in (0.0, -1.0, float("nan"), INF, 1e-31, 1e31):
        with pytest.raises(CocodError):
            ops.token_logprobs(ys, scale=bad)
    t = plan.order % D
    known = ops.token_logprobs(ys, t, top=3)
    g = gaussian(1, T * k)
    for call in (lambda: ops.token_logprobs_grad(ys, None, known, g), lambda: ops.token_logprobs_grad(ys, t, known, g[1:]), lambda: ops.token_logprobs_grad(ys, t, known, g.double()),
                 lambda: ops.token_logprobs_grad(ys, t, known, g, d_top=gaussian(1, T * k, 2)), lambda: ops.token_logprobs_grad(ys, t, known._replace(top_tokens=None), d_top=gaussian(1, T * k, 3)),
                 lambda: ops.token_logprobs_grad(ys, t, known._replace(entropy=None), d_entropy=g), lambda: ops.token_logprobs_grad(ys, t, known._replace(log_sum=None), g),
                 lambda: ops.token_logprobs_grad(ys, t, known, g, out=ys.bfloat16()), lambda: ops.token_logprobs_grad(ys[1:], t[1:], known, g[1:])):
        with pytest.raises(ValueError):
            call()
    ops.check()


# ------------------------------------------------------------------------------------------------------- log probabilities
def plain_logprobs(logits, tokens, top, scale):
    x = logits.double()
    y = x * scale
    most = y.amax(1, keepdim=True)
    dead = most[:, 0] == -INF
    t = y - torch.where(dead[:, None], 0.0, most)            # (relative to the largest: a row of the type's lowest value has a distribution, too)
    log_sum = torch.logsumexp(t, 1)
    z = log_sum + most[:, 0]
    lp = torch.where(dead[:, None], torch.full_like(y, -INF), t - log_sum[:, None])
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, torch.where(p.isnan(), p, 0.0)).sum(1)
    best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    got = [None if tokens is None else lp.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0], h, z, lp.gather(1, best), best]
    if tokens is not None:
        out = tokens < 0
        for a, fill in zip(got, (0, 0, 0, 0, -1)):
            a[out] = fill
    return got


def assert_logprobs(got, logits, tokens, top, scale):
    want = plain_logprobs(logits, tokens, top, scale)
    V = logits.shape[1]
    s = 19 * 2.0 ** -22 + (V / 128 + 64) * 2.0 ** -24
    z, finite = want[2], want[2].isfinite()
    most = (logits.double() * scale).masked_fill(~(logits.abs() < 1e30), 0).abs().amax(1)

    def close(a, b, bound, name):
        assert a.shape == b.shape, name
        same = (a.double() == b) | (a.isnan() & b.isnan())
        near = ((a.double() - b).abs() <= bound) & b.isfinite()
        assert (same | near).all(), f"{name}: worst {((a.double() - b).abs() / bound)[b.isfinite()].max()} of the bound"

    step = s + 2.0 ** -22 * (1 + torch.where(finite, z.abs(), 0.0))
    if tokens is not None:
        own = torch.where(want[0].isfinite(), want[0].abs(), 0.0)
        close(got.logp, want[0], step + 2.0 ** -22 * (own + 2 * most), "logp")
    close(got.entropy, want[1], s * (2 + math.log(V)) + 2.0 ** -23, "entropy")
    close(got.log_sum, z, step + 2.0 ** -23 * most, "log_sum")
    if top:
        assert torch.equal(got.top_tokens.long(), want[4])
        lp = torch.where(want[3].isfinite(), want[3].abs(), 0.0)
        close(got.top_logp, want[3], (step + 2.0 ** -22 * 2 * most)[:, None] + 2.0 ** -22 * lp, "top_logp")


LOGITS = [(1, 1, 1), (3, 2, 2), (5, 7, 3), (64, 31, 31), (17, 32, 32), (100, 64, 4), (33, 100, 20), (9, 257, 8), (21, 513, 32), (12, 1000, 5), (8, 1024, 32), (7, 1025, 32), (40, 1033, 20),
          (5, 2048, 32), (300, 4097, 3), (1, 8191, 32), (4, 50001, 20), (2, 131072, 32), (150, 33333, 1), (600, 5000, 0)]


@pytest.mark.parametrize("M,V,top", LOGITS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["plain", "masked", "far apart", "equal"])
def test_log_probabilities(ops, M, V, top, dtype, kind):
    x = gaussian(M + V, M, V, scale=2.0, dtype=dtype)
    scale = 1.0
    g = torch.Generator(device="cuda").manual_seed(V)
    if kind == "masked":                                    # all but few, or nothing at all
        keep = torch.rand(M, V, generator=g, device="cuda") < torch.rand(M, 1, generator=g, device="cuda") * 0.5
        x = x.masked_fill(~keep, -INF)
        x[::5] = x[::5].masked_fill(x[::5] == -INF, torch.finfo(dtype).min)
        x[M // 2] = -INF
        x[M // 3, :] = -INF
        x[M // 3, V // 2] = -3.0
    elif kind == "far apart":
        x, scale = x * 40, 0.7
    elif kind == "equal":
        x = (x / 3).round() * 0.0 + torch.randint(0, 2, (M, V), generator=g, device="cuda").to(dtype) * (torch.arange(M, device="cuda") % 3 == 0)[:, None]
        x[1::2] = -x[1::2]                                  # zeros of either sign
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    tokens[::7] = -1 if M > 7 else tokens[::7]
    assert_logprobs(ops.token_logprobs(x, tokens, top=top, scale=scale), x, tokens, top, scale)
    alone = ops.token_logprobs(x, top=top, scale=scale)
    assert alone.logp is None
    assert_logprobs(alone, x, None, top, scale)
    ops.check()


@pytest.mark.parametrize("V", [40, 3000, 20000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_alternatives_where_the_bound_is_of_no_use(ops, V, dtype):
    """Rows made so that few threads hold all large values, in every order, and rows with hundreds of values above all others."""
    M, top = 12, min(V, 32)
    x = torch.zeros(M, V, device="cuda")
    i = torch.arange(V, device="cuda")
    x[0], x[1] = i, -i.float()
    x[2] = (i % 8 == 3) * 5.0
    x[3] = (i % 512 == 17) * 5.0 + (i % 7) * 0.01
    x[4] = (i // 8 % 512 < 3) * (i % 200).float()
    x[5] = (i // 8 % 512 < 2) * 4.0
    x[6, -3:] = 1
    x[7, :3] = 1
    x[8] = (i // 4 % 512 < 5) * (1 + i.float() / V)
    x[9] = i // (V // 2)
    x[10] = -INF
    x[10, V // 3:V // 3 + 5] = i[:5].float()
    x[11] = torch.where(i % 64 < 20, 3.0, -INF)
    x = x.to(dtype)
    assert_logprobs(ops.token_logprobs(x, top=top), x, None, top, 1.0)
    wide = torch.full((M, V + 5), 99.0, dtype=dtype, device="cuda")
    for lead in range(6):                                   # any alignment: what lies beside the rows is not looked at
        wide.fill_(99.0)
        v = wide[:, lead:lead + V] if lead < 6 else wide
        v.copy_(x)
        a, b = ops.token_logprobs(v, top=top), ops.token_logprobs(x, top=top)
        assert torch.equal(a.top_tokens, b.top_tokens)
        assert_logprobs(a, x, None, top, 1.0)


@pytest.mark.parametrize("V", [50, 1500, 40000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_that_are_not_finite(ops, V, dtype):
    x = gaussian(1, 6, V, dtype=dtype)
    x[0, 7], x[1, V - 1], x[2, 0], x[2, 3], x[3, 5] = float("nan"), INF, INF, float("nan"), -float("nan")
    t = torch.full((6,), 9, dtype=torch.int32, device="cuda")
    t[3] = -1
    r = ops.token_logprobs(x, t, top=4)
    assert r.logp[:3].isnan().all() and r.entropy[:3].isnan().all() and r.log_sum[:3].isnan().all() and r.top_logp[:3].isnan().all()
    assert r.top_tokens[0, 0] == 7 and r.top_tokens[1, 0] == V - 1 and r.top_tokens[2, :2].tolist() == [3, 0]
    assert (r.top_tokens[3] == -1).all() and r.logp[3] == 0 and r.entropy[3] == 0 and r.log_sum[3] == 0 and (r.top_logp[3] == 0).all()
    assert r.logp[4:].isfinite().all() and r.entropy[4:].isfinite().all()
    d = ops.token_logprobs_grad(x, t, r, torch.ones(6, device="cuda"), torch.ones(6, device="cuda"))
    assert d[:3].isnan().any(1).all() and (d[3] == 0).all() and d[4:].isfinite().all()


def test_a_token_beyond_the_vocabulary_takes_no_part_and_is_reported(ops):
    from paper_1906_12043_b200.engine import CocodError
    for V in (60, 5000):
        x = gaussian(1, 3, V)
        t = torch.tensor([1, V, 2], dtype=torch.int32, device="cuda")
        r = ops.token_logprobs(x, t, top=2)
        with pytest.raises(CocodError):
            ops.check()
        assert r.logp[1] == 0 and (r.top_tokens[1] == -1).all() and r.logp[0] != 0
        d = ops.token_logprobs_grad(x, t, r, torch.ones(3, device="cuda"))
        assert (d[1] == 0).all() and d[0].any()
        with pytest.raises(CocodError):
            ops.check()
        known = r._replace(top_tokens=torch.tensor([[1, 2], [-1, -1], [5, V]], dtype=torch.int32, device="cuda"))
        g = torch.ones(3, 2, device="cuda")
        d = ops.token_logprobs_grad(x, None, known, d_top=g)
        with pytest.raises(CocodError):
            ops.check()
        assert (d[2].double().sum().abs() <= 1e-5) and d[2, 5] > 0


def plain_gradient(x, tokens, r, d_logp, d_entropy, d_top, scale):
    """(gradient, bound on the error of a result in fp32)"""
    z, h = r.log_sum.double()[:, None], r.entropy.double()[:, None]
    y = x.double() * scale
    dead = (z == -INF) | (tokens < 0)[:, None]
    lp = torch.where(dead, 0.0, y - z)
    p = lp.exp()
    given = torch.zeros_like(y)
    given.scatter_add_(1, tokens.clamp(min=0).long()[:, None], d_logp.double()[:, None])
    if d_top is not None:
        given.scatter_add_(1, r.top_tokens.clamp(min=0).long(), torch.where(r.top_tokens >= 0, d_top.double(), 0.0))
    every = given.sum(1, keepdim=True)
    size = d_logp.double().abs()[:, None] + (0 if d_top is None else d_top.double().abs().sum(1, keepdim=True))
    g = d_entropy.double()[:, None]
    inner = torch.where(p > 0, lp + h, 0.0)
    d = given - torch.where(p > 0, p * (every + g * inner), 0.0)
    a = 2.0 ** -22 * (1 + torch.where(y.isfinite(), y.abs(), 0.0) + z.abs())
    bound = p * ((2.0 ** -21 + a) * (size + g.abs() * inner.abs()) + g.abs() * (a + 2.0 ** -23 * (h + inner.abs()))) + 36 * 2.0 ** -24 * size * (given != 0) + 2.0 ** -100
    return torch.where(dead, 0.0, scale * d), torch.where(dead, 0.0, scale * (bound + 2.0 ** -23 * d.abs()))


@pytest.mark.parametrize("M,V,top", [(1, 1, 0), (3, 2, 2), (50, 64, 4), (9, 999, 0), (20, 1000, 8), (37, 8191, 0), (5, 50001, 20), (3, 131072, 32), (200, 4100, 1)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [False, True])
def test_gradient(ops, M, V, top, dtype, masked):
    x = gaussian(V, M, V, scale=2.0, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(M)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    if masked:
        x = x.masked_fill(torch.rand(M, V, generator=g, device="cuda") < 0.4, -INF)
        x[M // 2] = -INF
        if M > 2:
            tokens[0] = -1
    scale = 1.0 if M % 2 else 0.6
    r = ops.token_logprobs(x, tokens, top=top, scale=scale)
    d_logp, d_entropy = gaussian(1, M), gaussian(2, M)
    d_top = gaussian(3, M, top) if top else None
    if top > 2:                                             # the row's token among the alternatives, and one of them twice
        r.top_tokens[:, 1] = r.top_tokens[:, 0]
        r.top_tokens[:, 2] = torch.where(tokens >= 0, tokens, -1)
    want, bound = plain_gradient(x, tokens, r, d_logp, d_entropy, d_top, scale)
    got = ops.token_logprobs_grad(x, tokens, r, d_logp, d_entropy, d_top, scale=scale)
    assert got.dtype == dtype
    error, room = (got.double() - want).abs(), bound + half_step(dtype) * want.abs()
    assert (error <= room).all(), f"worst {(error / room.clamp(min=1e-300)).max()}"
    over = x.clone()
    assert ops.token_logprobs_grad(over, tokens, r, d_logp, d_entropy, d_top, scale=scale, out=over) is over
    assert torch.equal(over, got)
    whole = torch.full((M + 2, V + 9), 7.0, dtype=dtype, device="cuda")       # another alignment than the logits'
    ops.token_logprobs_grad(x, tokens, r, d_logp, d_entropy, d_top, scale=scale, out=whole[1:-1, 3:3 + V])
    assert torch.equal(whole[1:-1, 3:3 + V], got)
    whole[1:-1, 3:3 + V] = 7
    assert (whole == 7).all()
    ops.check()


def test_gradient_against_differences(ops):
    """The definition's values in 64 bits at two points on either side."""
    M, V, scale = 4, 30, 0.8
    x = gaussian(1, M, V).double()
    tokens = torch.tensor([3, 0, 29, 7], dtype=torch.int32, device="cuda")
    a, b, c = (gaussian(s, M).double() for s in (2, 3, 4))

    def value(x):
        r = plain_logprobs(x, tokens, 2, scale)
        return (a * r[0] + b * r[1] + c * r[3][:, 1]).sum()

    r = ops.token_logprobs(x.float(), tokens, top=2, scale=scale)
    got = ops.token_logprobs_grad(x.float(), tokens, r, a.float(), b.float(), torch.stack([torch.zeros_like(c), c], 1).float(), scale=scale).double()
    for row, col in ((0, 3), (0, 4), (1, 0), (2, 29), (3, 8), (3, int(r.top_tokens[3, 1]))):
        up, down = x.clone(), x.clone()
        up[row, col] += 1e-5
        down[row, col] -= 1e-5
        assert abs(float(value(up) - value(down)) / 2e-5 - float(got[row, col])) <= 1e-5


def test_more_than_2_to_the_31_logits(ops):
    M, V = 40000, 65536
    x = torch.empty(M, V, dtype=torch.bfloat16, device="cuda")
    for a in range(0, M, 4000):
        x[a:a + 4000] = gaussian(a, 4000, V, dtype=torch.bfloat16)
    t = torch.randint(0, V, (M,), device="cuda", dtype=torch.int32)
    r = ops.token_logprobs(x, t, top=2)
    last = slice(M - 500, M)
    assert_logprobs(type(r)(*(v[last] for v in r)), x[last], t[last], 2, 1.0)
    g = torch.ones(M, device="cuda")
    want = ops.token_logprobs_grad(x[last], t[last], type(r)(*(v[last].contiguous() for v in r)), g[last])
    ops.token_logprobs_grad(x, t, r, g, out=x)
    assert torch.equal(x[last], want)
    ops.check()


def test_no_rows_at_all(ops):
    for k, E in ((1, 3), (4, 9)):
        plan = ops.expert_sort(torch.empty(0, k, dtype=torch.int32, device="cuda"), E)
        assert plan.offsets.tolist() == [0] * (E + 1) and plan.counts.tolist() == [0] * E and plan.order.shape == (0,) and plan.place.shape == (0, k)
        x, w = torch.empty(0, 24, device="cuda"), torch.empty(0, k, device="cuda")
        rows = ops.expert_rows(x, plan)
        assert rows.shape == (0, 24) and ops.expert_rows_grad(rows, plan).shape == (0, 24) and ops.expert_join(rows, plan, w).shape == (0, 24)
        d, dw = ops.expert_join_grad(x, rows, plan, w)
        assert d.shape == (0, 24) and dw.shape == (0, k)
    for V in (5, 500, 50000):
        x, t = torch.empty(0, V, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
        r = ops.token_logprobs(x, t, top=3)
        assert r.logp.shape == r.entropy.shape == r.log_sum.shape == (0,) and r.top_logp.shape == r.top_tokens.shape == (0, 3)
        assert ops.token_logprobs_grad(x, t, r, torch.empty(0, device="cuda")).shape == (0, V)
    ops.check()


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e6, 1e30])
def test_scales_far_from_one(ops, scale):
    """The softmax of scale * logits, from all equal to a single one."""
    for V in (60, 3000, 40000):
        x = gaussian(V, 5, V)
        x[1, ::2] = -INF
        x[2, 3] = x[2].max()
        t = torch.full((5,), 3, dtype=torch.int32, device="cuda")
        assert_logprobs(ops.token_logprobs(x, t, top=4, scale=scale), x, t, 4, scale)
    ops.check()


def test_two_streams_at_once(ops):
    """Calls that share nothing but the report of errors."""
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    x, y = gaussian(1, 300, 30000, dtype=torch.bfloat16), gaussian(2, 300, 30000, dtype=torch.bfloat16)
    e, f = choices(3, 9000, 4, 64), choices(4, 9000, 4, 64)
    want = [ops.token_logprobs(x, top=5), ops.token_logprobs(y, top=5), ops.expert_sort(e, 64), ops.expert_sort(f, 64)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for s, logits, experts in ((a, x, e), (b, y, f)):
            with torch.cuda.stream(s):
                got.append((ops.token_logprobs(logits, top=5), ops.expert_sort(experts, 64)))
    torch.cuda.synchronize()
    for i, (r, plan) in enumerate(got):
        assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(r, want[i % 2]))
        assert all(torch.equal(p, q) for p, q in zip(plan, want[2 + i % 2]))


def test_captured_and_replayed_and_on_another_stream(ops):
    """One graph of a whole way there and back: the same bits as the calls, and new ones for new inputs."""
    T, k, E, D, V = 600, 2, 16, 128, 16
    logits, x, dy = gaussian(1, T, V), gaussian(2, T, D), gaussian(3, T, D)

    def way():
        r = ops.token_logprobs(logits, top=k)
        plan = ops.expert_sort(r.top_tokens, E)
        w = r.top_logp.exp()
        rows = ops.expert_rows(x, plan)
        y = ops.expert_join(rows, plan, w)
        drows, dw = ops.expert_join_grad(dy, rows, plan, w)
        dl = ops.token_logprobs_grad(logits, None, r, d_top=dw * w)
        return y, ops.expert_rows_grad(drows, plan), dl, plan.order

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        way()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = way()
    torch.cuda.current_stream().wait_stream(s)
    for seed in (5, 6):
        logits.copy_(gaussian(seed, T, V))
        x.copy_(gaussian(seed + 10, T, D))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, way()))
    ops.check()


def test_the_same_bits_every_time(ops):
    x, t = gaussian(1, 50, 30000, dtype=torch.bfloat16), torch.arange(50, dtype=torch.int32, device="cuda")
    first = ops.token_logprobs(x, t, top=20)
    plan = ops.expert_sort(choices(1, 5000, 4, 64), 64)
    ys, dy, w = gaussian(2, 20000, 256), gaussian(3, 5000, 256), gaussian(4, 5000, 4)
    grads = ops.expert_join_grad(dy, ys, plan, w)
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, ops.token_logprobs(x, t, top=20)))
        assert all(torch.equal(a, b) for a, b in zip(grads, ops.expert_join_grad(dy, ys, plan, w)))


def spread(x, scale):
    """In 64 bits, without cancellation: what all terms but the largest add up to, relative to it; the same weighted with their distances from it; and the sum over the
    terms of e^-d (2^-20 + 8 * 2^-24 d / ln 2) and of d times that."""
    y = x.double() * scale
    most, at = y.max(1, keepdim=True)
    d = most - y                                             # (distances in natural units)
    e = torch.exp(-d)
    e.scatter_(1, at, 0.0)
    near = torch.where(e > 0, d, 0.0)
    each = e * (2.0 ** -20 + 8 * 2.0 ** -24 * near / math.log(2))
    return e.sum(1), (e * near).sum(1), each.sum(1), (near * each).sum(1), d


@pytest.mark.parametrize("V", [257, 1000, 4000, 9001, 20000, 40000, 65536, 128256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M", [5, 230])
@pytest.mark.parametrize("scale", [1.0, 0.7])
def test_confident_rows(ops, V, dtype, M, scale):
    """Rows with a logit far above the others, wherever it lies: log probabilities are not above 0 and entropies not below, and both are as near to those of 64 bits as
    sums of the other terms allow.

    Let O be the sum of all terms but the largest, relative to it.  A term at distance d is off by a relative 2^-20 (the exponential and the factors of up to four changes of
    reference, 2^-22 each at most, the rounding of scale log2 e) and 8 * 2^-24 d / ln 2 (the roundings of its exponent and of the changes').  Sums add (V / 128 + 64) * 2^-24 of O.
    The largest term is exact, but for the other values of its batch, at most 17 of which are added to it and rounded with it: 18 * 2^-24 * (1 + O).  So log (1 + O) is off by
    at most E = these three over 1 + O, and the entropy log (1 + O) + D / (1 + O), D the terms times their distances, by E + D / (1 + O) E + the errors of D's terms, each of
    which has another 2^-23, the sums' of D, and 18 * 2^-24 * 2^-8 for the largest term's exponent, which is a rounding of at most 2^-8.  Results: 2^-22 of themselves."""
    x = gaussian(V + M, M, V, scale=2.0, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(V)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    far = (20 + 25 * torch.rand(M, generator=g, device="cuda")).to(dtype)
    x.scatter_(1, tokens.long()[:, None], far[:, None])
    x[0] = torch.linspace(-50, 10, V).to(dtype)              # (every batch's largest exceeds all before)
    x[1] = torch.linspace(10, -50, V).to(dtype)
    if M > 5:
        x[2, V // 3] = x[2].max()                            # (twice)
        x[3, ::3] = -INF
    tokens[4] = (tokens[4] + 1) % V                          # (not the confident token)
    O, D, each, weighted, d = spread(x, scale)
    sums = (V / 128 + 64) * 2.0 ** -24
    E = (each + sums * O) / (1 + O) + 18 * 2.0 ** -24
    H = torch.log1p(O) + D / (1 + O)
    lp = -d.gather(1, tokens.long()[:, None])[:, 0] - torch.log1p(O)
    for top in (0, 3):
        r = ops.token_logprobs(x, tokens, top=top, scale=scale)
        assert (r.logp <= 0).all() and (r.entropy >= 0).all()
        error = torch.where(r.logp.double() == lp, 0.0, (r.logp.double() - lp).abs())      # (a masked token: -inf)
        room = E + 2.0 ** -22 * lp.abs()
        assert (error <= room).all(), f"log p: worst {(error / room).max()} of the bound"
        error = (r.entropy.double() - H).abs()
        room = E + (D * E + weighted + (2.0 ** -23 + sums) * D) / (1 + O) + 18 * 2.0 ** -32 + 2.0 ** -22 * H
        assert (error <= room).all(), f"entropy: worst {(error / room).max()} of the bound"
        if top:
            assert (r.top_logp <= 0).all()
            assert torch.equal(r.top_tokens.long(), torch.sort(x.double(), dim=1, descending=True, stable=True).indices[:, :top])
    ops.check()


def test_a_result_that_is_given_is_an_operation_in_place_for_autograd(ops):
    """Every out= and dw=: what autograd kept of the tensor is not used for a backward pass after it was written."""
    M, k, n = 32, 64, 48
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    x, w, dy = gaussian(1, M, k, dtype=torch.bfloat16), gaussian(2, 1, n, k, dtype=torch.bfloat16), gaussian(3, M, n, dtype=torch.bfloat16)
    packed, labels, experts = ops.act_pack(x), torch.zeros(M, dtype=torch.int32, device="cuda"), choices(1, M, 2, 4)
    plan, p = ops.expert_sort(experts, 4), gaussian(4, M, 2)
    rows = ops.expert_rows(x, plan)
    known = ops.token_logprobs(dy, labels)
    calls = [(lambda out: ops.grouped_forward(x, w, off, out=out), dy), (lambda out: ops.grouped_input_grad(dy, w, off, out=out), x),
             (lambda out: ops.grouped_weight_grad(dy, x, off, out=out), w), (lambda out: ops.grouped_weight_grad(dy, packed, off, out=out), w),
             (lambda out: ops.act_unpack(packed, out=out), x), (lambda out: ops.act_relu_grad(x, packed, out=out), x),
             (lambda out: ops.vocab_loss_grad(x, w, labels, off, dw=out), w), (lambda out: ops.expert_rows(x, plan, out=out), rows),
             (lambda out: ops.expert_rows_grad(rows, plan, out=out), x), (lambda out: ops.expert_join(rows, plan, p, out=out), x),
             (lambda out: ops.expert_join_grad(x, rows, plan, p, out=out), rows), (lambda out: ops.token_logprobs_grad(dy, labels, known, gaussian(1, M), out=out), dy)]
    for call, like in calls:
        leaf = torch.zeros_like(like, requires_grad=True)
        kept = leaf.exp()                                    # (whose own value is its gradient)
        whole = kept.sum()
        call(kept.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            whole.backward()
        with torch.inference_mode():
            call(torch.zeros_like(like))
    logits = torch.zeros_like(dy, requires_grad=True).exp()
    ops.token_logprobs_grad(logits.detach(), labels, known, gaussian(1, M), out=logits.detach())
    assert logits._version == 1
    ops.check()


def test_new_results_are_seen_by_dispatch_modes_and_filled_where_torch_fills_them(ops):
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __init__(self):
            super().__init__()
            self.names = []

        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            self.names.append(str(func))
            return func(*args, **(kwargs or {}))

    M, k, n = 32, 64, 48
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    x, w = gaussian(1, M, k, dtype=torch.bfloat16), gaussian(2, 1, n, k, dtype=torch.bfloat16)
    plan = ops.expert_sort(choices(1, M, 2, 4), 4)
    place = plan.place.clone()
    place = torch.where(place == 2 * M - 1, place.flip(1), place)      # (a row that no place names is not written; its token has its other row twice)
    calls = [lambda: ops.grouped_forward(x, w, off), lambda: ops.expert_rows(x, plan._replace(place=place))]
    before = [call() for call in calls]
    with Seen() as seen:
        for call in calls:
            call()
        ops.token_logprobs(x, top=2)
        ops.expert_sort(plan.place.abs() % 4, 4)
    assert sum("aten.empty" in name for name in seen.names) >= 4
    was = torch.are_deterministic_algorithms_enabled(), torch.utils.deterministic.fill_uninitialized_memory
    try:
        torch.use_deterministic_algorithms(True, warn_only=True)
        torch.utils.deterministic.fill_uninitialized_memory = True
        torch.cuda.empty_cache()
        y, rows = (call() for call in calls)
        assert torch.equal(y, before[0]) and rows[-1].isnan().all() and torch.equal(rows[:-1], before[1][:-1])
    finally:
        torch.use_deterministic_algorithms(was[0])
        torch.utils.deterministic.fill_uninitialized_memory = was[1]
    ops.check()


def test_a_result_does_not_lie_on_any_operand(ops):
    """... the small ones among them, which threads still read when others have written."""
    T, k, E = 64, 8, 16
    plan = ops.expert_sort(choices(1, T, k, E), E)
    x, ys, w = gaussian(1, T, k), gaussian(2, T * k, k), gaussian(3, T, k)
    place = plan.place.view(torch.float32)
    wide = torch.zeros(T * k, k, device="cuda")
    on_rows = wide[:T].copy_(w)
    kept = [t.clone() for t in (plan.place, w)]
    wide_plan = plan._replace(place=wide.view(torch.int32)[T:2 * T].copy_(plan.place))
    for call in (lambda: ops.expert_join(ys, plan, w, out=w), lambda: ops.expert_join(ys, plan, w, out=place), lambda: ops.expert_rows_grad(ys, plan, out=place),
                 lambda: ops.expert_join_grad(x, ys, plan, on_rows, out=wide), lambda: ops.expert_join_grad(x, ys, wide_plan, w, out=wide),
                 lambda: ops.expert_rows(x, wide_plan, out=wide)):
        with pytest.raises(ValueError, match="lies on"):
            call()
    M, V = 12, 20
    logits, all_ = gaussian(4, M, V), torch.zeros(M, V, device="cuda")
    t = torch.zeros(M, dtype=torch.int32, device="cuda")
    known, g, d_top = ops.token_logprobs(logits, t, top=2), gaussian(5, M), gaussian(6, M, 2)

    def inside(v):                                           # (the same values somewhere in the result)
        return all_.view(v.dtype).view(-1)[7:7 + v.numel()].view(v.shape).copy_(v)

    for call in (lambda: ops.token_logprobs_grad(logits, inside(t), known, g, out=all_), lambda: ops.token_logprobs_grad(logits, t, known, inside(g), out=all_),
                 lambda: ops.token_logprobs_grad(logits, t, known, d_entropy=inside(g), out=all_), lambda: ops.token_logprobs_grad(logits, t, known, d_top=inside(d_top), out=all_),
                 lambda: ops.token_logprobs_grad(logits, t, known._replace(log_sum=inside(known.log_sum)), g, out=all_),
                 lambda: ops.token_logprobs_grad(logits, t, known._replace(entropy=inside(known.entropy)), d_entropy=g, out=all_),
                 lambda: ops.token_logprobs_grad(logits, t, known._replace(top_tokens=inside(known.top_tokens)), d_top=d_top, out=all_)):
        with pytest.raises(ValueError, match="lies on"):
            call()
    assert all(torch.equal(a, b) for a, b in zip(kept, (plan.place, w)))
    ops.check()


# ------------------------------------------------------------------------------------------------------- the forms that large batches take
@pytest.mark.parametrize("T,k,D", [(2500, 1, 512), (20000, 1, 64), (2500, 2, 1024), (1300, 2, 768), (6000, 1, 1027), (9000, 2, 520), (3000, 1, 2048), (1500, 5, 1032), (700, 12, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_joins_of_large_batches(ops, T, k, D, dtype):
    """Enough rows for every SM: the forms for one and two choices with full and with ragged widths, and the gradient's; the same bounds as above."""
    E = 32
    plan = ops.expert_sort(choices(T, T, k, E, 0.1), E)
    there = plan.place >= 0
    at = torch.where(there, plan.place, ~plan.place).long()
    ys, dy, w = gaussian(2, T * k, D, dtype=dtype), gaussian(3, T, D, dtype=dtype), gaussian(4, T, k)
    ys[at[~there]] = float("nan")
    wide = torch.where(there[..., None], ys.double()[at], 0.0)
    for out_dtype in (torch.bfloat16, torch.float32):
        for f, got in ((w.double(), ops.expert_join(ys, plan, w, out_dtype=out_dtype)), (torch.ones_like(w).double(), ops.expert_rows_grad(ys, plan, out_dtype=out_dtype))):
            y, size = (f[..., None] * wide).sum(1), (f[..., None] * wide).abs().sum(1)
            assert ((got.double() - y).abs() <= half_step(out_dtype) * y.abs() + 1.01 * (k + 1) * 2.0 ** -24 * size).all()
    drows, dw = ops.expert_join_grad(dy, ys, plan, w)
    back = torch.zeros(T * k, D, dtype=torch.float64, device="cuda")
    back[at[there]] = (w.double()[..., None] * dy.double()[:, None])[there]
    assert ((drows.double() - back).abs() <= 1.01 * (half_step(dtype) + 2.0 ** -24) * back.abs()).all() and (drows[at[~there]] == 0).all()
    products = wide * dy.double()[:, None]
    assert ((dw.double() - products.sum(2)).abs() <= (D / 32 + 16) * 2.0 ** -24 * products.abs().sum(2)).all() and (dw[~there] == 0).all()
    ops.check()


@pytest.mark.parametrize("M,V", [(2000, 300), (2000, 4000), (2000, 9001), (1300, 12000), (1200, 20000), (650, 47999), (400, 50001), (200, 128256), (160, 300000)])
@pytest.mark.parametrize("top", [0, 5, 32])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["plain", "masked", "coarse"])
def test_log_probabilities_of_large_batches(ops, M, V, top, dtype, kind):
    """Enough rows for every SM: 32, 64, 128 and 256 threads a row, each with more batches than it has slots among the longest rows; the same bounds as above."""
    x = gaussian(M + V, M, V, scale=2.0, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(V)
    if kind == "masked":
        x = x.masked_fill(torch.rand(M, V, generator=g, device="cuda") < torch.rand(M, 1, generator=g, device="cuda"), -INF)
        x[3] = -INF
        x[4, :-2] = -INF
    elif kind == "coarse":                                  # many equal values: the lowest index first
        x = (x * 2).round() / 2
        x[5] = 1.0
        x[6, V // 2:] = 40.0
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    tokens[::9] = -1
    for a in range(0, M, 400):                              # (a part of the rows at a time in 64 bits)
        if a == 0:
            r = ops.token_logprobs(x, tokens, top=top)
        part = type(r)(*(None if v is None else v[a:a + 400] for v in r))
        assert_logprobs(part, x[a:a + 400], tokens[a:a + 400], top, 1.0)
    ops.check()
