"""The language-model operators (lm.LMOps) against plain implementations in 64 bits.

Tolerances, derived before the first run:

* bf16 result of an fp32 sum: half a unit in the last place of bf16, at most 2^-8 of the value (8 significant bits), plus the sum's error.
* fp32 sum of L products of bf16 (exact in fp32): the tensor cores cut off bits, at most one unit of 2^-23 of the running sum's
  magnitude for every step of 16, and the parts of at most 512 (32 steps) are added with rounding; |error| <= 40 * 2^-23 * sum |a b|
  + (parts) * 2^-24 * (largest partial sum).  Both are below 2^-17 * sum |a b| for the lengths here.  For bf16 results, whose sums are not
  cut into parts, L / 16 + 8 steps: 2^-8 * |result| + (L / 16 + 8) * 2^-23 * sum |a b|.
* vocabulary: a logit's error is (D / 16 + 8) * 2^-23 * |h| |w| =: d; the loss moves by at most 2 d + 2^-20 * (1 + loss); a term of dx
  carries one bf16 rounding (2^-8) + 2 d, a term of dw three (the exponential, the scaled row, and the factor that makes up for the
  rounding of the label's entry), and the result one more rounding.
* 8 bits: the definition is exact, so equality.
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


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


def offsets_of(sizes):
    o = [0]
    for s in sizes:
        o.append(o[-1] + s)
    return torch.tensor(o, dtype=torch.int32, device="cuda"), [slice(a, b) for a, b in zip(o, o[1:])]


def gaussian(seed, *shape, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).bfloat16()


def assert_sum(got, want, absolute, length):
    """got: the result of a sum of `length` products whose magnitudes add up to `absolute`."""
    if got.dtype == torch.float32:
        bound = 2.0 ** -17 * absolute
    else:
        bound = 2.0 ** -8 * want.abs() + (length / 16 + 8) * 2.0 ** -23 * absolute * 1.01 + 1e-38
    bad = (got.double() - want).abs() > bound
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} outside, worst {((got.double() - want).abs() / bound.clamp(min=1e-300)).max():.3f} of the bound"


def products(x, w, dy, spans):
    d = torch.float64
    y = torch.cat([x[s].to(d) @ w[g].to(d).T for g, s in enumerate(spans)])
    ya = torch.cat([x[s].to(d).abs() @ w[g].to(d).abs().T for g, s in enumerate(spans)])
    dx = torch.cat([dy[s].to(d) @ w[g].to(d) for g, s in enumerate(spans)])
    dxa = torch.cat([dy[s].to(d).abs() @ w[g].to(d).abs() for g, s in enumerate(spans)])
    dw = torch.stack([dy[s].to(d).T @ x[s].to(d) for s in spans])
    dwa = torch.stack([dy[s].to(d).abs().T @ x[s].to(d).abs() for s in spans])
    return (y, ya), (dx, dxa), (dw, dwa)


SHAPES = [
    # sizes of the groups, n, k
    ([1], 8, 8),
    ([1, 0, 1], 16, 72),
    ([37], 136, 64),
    ([127, 1, 128, 129], 128, 200),
    ([0, 0, 256, 0], 512, 264),
    ([255, 257], 264, 512),
    ([700, 0, 5, 900, 31], 1024, 784),
    ([3] * 70, 64, 128),                       # more groups than a warp looks at together
    ([2049], 520, 2056),
    ([4096, 100], 256, 1032),
]


@pytest.mark.parametrize("sizes,n,k", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_products_by_group(ops, sizes, n, k, dtype):
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    x, w, dy = gaussian(1, M, k), gaussian(2, G, n, k, scale=k ** -0.5), gaussian(3, M, n)
    (y, ya), (dx, dxa), (dw, dwa) = products(x, w, dy, spans)
    assert_sum(ops.grouped_forward(x, w, off, out_dtype=dtype), y, ya, k)
    assert_sum(ops.grouped_input_grad(dy, w, off, out_dtype=dtype), dx, dxa, n)
    assert_sum(ops.grouped_weight_grad(dy, x, off, out_dtype=dtype), dw, dwa, max(sizes))
    ops.check()


@pytest.mark.parametrize("sizes,n,k", [([300, 0, 213], 136, 72), ([64] * 5, 256, 520), ([1500], 768, 384)])
def test_views_of_the_workers_state(ops, sizes, n, k):
    """Weights, results and rows as views: rows of a larger matrix, groups a whole model apart."""
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    P = n * k + 64 + k
    P = (P + 63) // 64 * 64
    x = gaussian(1, M, k + 24)[:, 8:8 + k]
    dy = gaussian(3, M, n + 8)[:, :n]
    w = gaussian(2, G, P, scale=k ** -0.5)[:, 64:64 + n * k].view(G, n, k)
    (y, ya), (dx, dxa), (dw, dwa) = products(x, w, dy, spans)
    for dtype in (torch.bfloat16, torch.float32):
        grads = torch.full((G, P), 7.0, device="cuda", dtype=dtype)
        big = torch.full((M, n + 16), 7.0, device="cuda", dtype=dtype)
        got = ops.grouped_weight_grad(dy, x, off, out=grads[:, 64:64 + n * k].view(G, n, k))
        assert_sum(got, dw, dwa, max(sizes))
        assert (grads[:, :64] == 7).all() and (grads[:, 64 + n * k:] == 7).all()
        assert_sum(ops.grouped_forward(x, w, off, out=big[:, 8:8 + n]), y, ya, k)
        assert (big[:, :8] == 7).all() and (big[:, 8 + n:] == 7).all()
    assert_sum(ops.grouped_input_grad(dy, w, off), dx, dxa, n)


@pytest.mark.parametrize("sizes,n,k", [([6294, 100, 6294], 592, 392), ([20000], 136, 72), ([3000, 9000], 264, 520), ([40, 0, 12000], 200, 1032)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_reductions_with_few_results(ops, sizes, n, k, dtype):
    """Tiles whose reduction is cut into parts, at widths that end inside a tile: every group's matrix is complete and nothing beside it is
    written."""
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    P = n * k + 512
    x, dy = gaussian(1, M, k), gaussian(3, M, n)
    want = torch.stack([dy[s].double().T @ x[s].double() for s in spans])
    size = torch.stack([dy[s].double().abs().T @ x[s].double().abs() for s in spans])
    grads = torch.full((G + 1, P), 7.0, device="cuda", dtype=dtype)
    out = torch.as_strided(grads, (G, n, k), (P, k, 1), 256)
    for a in (x, ops.act_pack(x)):
        grads.fill_(7.0)
        got = ops.grouped_weight_grad(dy, a, off, out=out)
        if a is x:
            assert_sum(got, want, size, max(sizes))
        else:
            kept = ops.act_unpack(a)
            assert_sum(got, torch.stack([dy[s].double().T @ kept[s].double() for s in spans]), size * 1.02 + 1e-3, max(sizes))
        assert (grads[0, :256] == 7).all() and (grads[G] == 7).all() and (grads[:G, 256 + n * k:] == 7).all()
        assert (grads[1:G, :256] == 7).all()
    # and the rows form: a deep product with few rows
    w = gaussian(2, G, 264, M // 8 * 8, scale=0.02)
    few, few_spans = offsets_of([3, 30] + [5] * (G - 2) if G > 1 else [37])
    r = int(few[-1])
    deep = gaussian(4, r, w.shape[2])
    y = torch.full((r + 2, 272), 7.0, device="cuda", dtype=dtype)
    ops.grouped_forward(deep, w, few, out=y[1:-1, :264])
    yw = torch.cat([deep[s].double() @ w[g].double().T for g, s in enumerate(few_spans)])
    ya = torch.cat([deep[s].double().abs() @ w[g].double().abs().T for g, s in enumerate(few_spans)])
    assert_sum(y[1:-1, :264], yw, ya, w.shape[2])
    assert (y[0] == 7).all() and (y[-1] == 7).all() and (y[:, 264:] == 7).all()
    dx = ops.grouped_input_grad(gaussian(5, r, 264), gaussian(6, G, 264, 4096, scale=0.1), few)
    assert torch.isfinite(dx.float()).all()


def test_other_groups_values_never_leak(ops):
    """NaN and infinities in one group's rows and weights stay in that group's results."""
    sizes = [130, 61, 7, 300]
    off, spans = offsets_of(sizes)
    x, w, dy = gaussian(1, 498, 192), gaussian(2, 4, 264, 192), gaussian(3, 498, 264)
    x[spans[1]] = float("nan")
    dy[spans[1]] = float("inf")
    w[1] = float("nan")
    y, dx, dw = ops.grouped_forward(x, w, off), ops.grouped_input_grad(dy, w, off), ops.grouped_weight_grad(dy, x, off)
    for g, s in enumerate(spans):
        assert torch.isfinite(y[s]).all() == (g != 1) and torch.isfinite(dx[s]).all() == (g != 1)
        assert torch.isfinite(dw[g]).all() == (g != 1)


def test_no_rows_and_empty_groups(ops):
    off, _ = offsets_of([0, 0, 0])
    w = gaussian(2, 3, 64, 128)
    x, dy = torch.empty(0, 128, device="cuda", dtype=torch.bfloat16), torch.empty(0, 64, device="cuda", dtype=torch.bfloat16)
    assert ops.grouped_forward(x, w, off).shape == (0, 64) and ops.grouped_input_grad(dy, w, off).shape == (0, 128)
    out = torch.full((3, 64, 128), 5.0, device="cuda")
    assert (ops.grouped_weight_grad(dy, x, off, out=out) == 0).all()
    loss, row_loss, dx, dw = ops.vocab_loss_grad(x, w, torch.empty(0, dtype=torch.int32, device="cuda"), off)
    assert (loss == 0).all() and row_loss.shape == (0,) and dx.shape == (0, 128) and (dw == 0).all()


def test_products_repeat_bit_for_bit_and_on_another_stream(ops):
    off, _ = offsets_of([900, 20, 1128])
    x, w, dy = gaussian(1, 2048, 512), gaussian(2, 3, 640, 512), gaussian(3, 2048, 640)
    want = ops.grouped_forward(x, w, off), ops.grouped_input_grad(dy, w, off), ops.grouped_weight_grad(dy, x, off)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ops.grouped_forward(x, w, off), ops.grouped_input_grad(dy, w, off), ops.grouped_weight_grad(dy, x, off)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_weight_gradient_is_the_forward_products_derivative(ops):
    """d <y, dy> / d w and d x against differences: the forward product is linear, so that a step of 2^-3 is exact but for rounding."""
    off, spans = offsets_of([40, 25])
    x, w, dy = gaussian(1, 65, 64), gaussian(2, 2, 72, 64, scale=0.125), gaussian(3, 65, 72)
    dw, dx = ops.grouped_weight_grad(dy, x, off), ops.grouped_input_grad(dy, w, off, out_dtype=torch.float32)
    base = (ops.grouped_forward(x, w, off, out_dtype=torch.float32).double() * dy.double()).sum()
    for g, j, i in ((0, 0, 0), (0, 71, 63), (1, 13, 40)):
        w2 = w.clone()
        w2[g, j, i] += 4.0
        step = float(w2[g, j, i].double() - w[g, j, i].double())
        diff = ((ops.grouped_forward(x, w2, off, out_dtype=torch.float32).double() * dy.double()).sum() - base) / step
        # each of the two sums: 65 * 72 values, |y dy| of order 3, each y off by 2^-17 * sum |x w| (about 5)
        assert abs(float(diff) - float(dw[g, j, i])) <= 2 * 65 * 72 * 3 * 2.0 ** -17 * 5 / step
    for m, i in ((0, 0), (64, 63), (40, 7)):
        x2 = x.clone()
        x2[m, i] += 4.0
        step = float(x2[m, i].double() - x[m, i].double())
        diff = ((ops.grouped_forward(x2, w, off, out_dtype=torch.float32).double() * dy.double()).sum() - base) / step
        assert abs(float(diff) - float(dx[m, i])) <= 2 * 65 * 72 * 3 * 2.0 ** -17 * 5 / step


def test_products_replayed_from_a_graph(ops):
    off, spans = offsets_of([333, 0, 179])
    x, w, dy = gaussian(1, 512, 256), gaussian(2, 3, 384, 256), gaussian(3, 512, 384)
    y, dw = torch.empty(512, 384, device="cuda", dtype=torch.bfloat16), torch.empty(3, 384, 256, device="cuda")
    ops.grouped_forward(x, w, off, out=y), ops.grouped_weight_grad(dy, x, off, out=dw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ops.grouped_forward(x, w, off, out=y)
        ops.grouped_weight_grad(dy, x, off, out=dw)
    x.copy_(gaussian(7, 512, 256))
    off2, spans2 = offsets_of([100, 200, 212])
    off.copy_(off2)                              # the division of the rows is read on the device
    graph.replay()
    torch.cuda.synchronize()
    (yw, ya), _, (dww, dwa) = products(x, w, dy, spans2)
    assert_sum(y, yw, ya, 256)
    assert_sum(dw, dww, dwa, 512)


# ------------------------------------------------------------------------------------------------------- 8 bits
def pack_reference(x):
    """q and e from the definition, in Python's exact arithmetic by way of float64 (powers of two and bf16 values are exact)."""
    M, k = x.shape
    v = x.double().cpu()
    q, e = torch.zeros(M, k, dtype=torch.int64), torch.zeros(-(-k // 128), M, dtype=torch.int64)
    for b in range(e.shape[0]):
        part = v[:, 128 * b:128 * (b + 1)]
        finite = torch.isfinite(part)
        amax = torch.where(finite, part.abs(), 0.0).amax(1)
        for m in range(M):
            u = -126
            while amax[m].item() > 127 * 2.0 ** u:
                u += 1
            e[b, m] = u + 127
            for j in range(part.shape[1]):
                a = part[m, j].item()
                if not math.isfinite(a):
                    q[m, 128 * b + j] = -128
                    e[b, m] = 255
                elif a != 0:
                    n = max(1, round(abs(a) * 2.0 ** -u))       # Python rounds half to even
                    if n * 2.0 ** u >= 2.0 ** 128:
                        n -= 1                                    # bf16 ends there
                    q[m, 128 * b + j] = int(math.copysign(n, a))
    return q, e


@pytest.mark.parametrize("M,k", [(1, 1), (1, 8), (3, 127), (33, 128), (5, 129), (64, 200), (31, 16), (2, 1000)])
@pytest.mark.parametrize("kind", ["gaussian", "relu", "wide"])
def test_pack_is_its_definition(ops, M, k, kind):
    x = gaussian(M * k, M, k)
    if kind == "relu":
        x = x.clamp(min=0)
    if kind == "wide":
        x = (x.float() * torch.exp2(torch.randint(-140, 120, (M, k), generator=torch.Generator().manual_seed(1)).float().cuda())).bfloat16()
        if k > 5:
            x[0, 0], x[0, 1], x[0, k - 1] = float("inf"), float("nan"), float("-inf")
        if M > 1:
            x[1] = 0
    p = ops.act_pack(x)
    q, e = pack_reference(x)
    assert torch.equal(p.scales.long().cpu(), e)
    assert torch.equal(p.q.long().cpu(), q)
    y = ops.act_unpack(p)
    unit = torch.where(e == 255, float("nan"), torch.exp2(e.double() - 127)).T.repeat_interleave(128, 1)[:, :k]
    want = q.double() * unit
    assert torch.equal(torch.nan_to_num(y.double().cpu(), nan=-1e30), torch.nan_to_num(want, nan=-1e30))


def test_pack_at_the_end_of_bf16(ops):
    top = torch.finfo(torch.bfloat16).max
    x = torch.tensor([[top, -top, top / 2, 1.0, 0.0, 2.0 ** -133, -2.0 ** -126, 3e38]], device="cuda").bfloat16()
    p = ops.act_pack(x)
    q, e = pack_reference(x)
    assert torch.equal(p.q.long().cpu(), q) and torch.equal(p.scales.long().cpu(), e)
    assert torch.isfinite(ops.act_unpack(p).float()).all()
    tiny = torch.tensor([[2.0 ** -133, -2.0 ** -130, 0.0, 2.0 ** -127]], device="cuda").bfloat16()
    p = ops.act_pack(tiny)
    q, e = pack_reference(tiny)
    assert torch.equal(p.q.long().cpu(), q) and torch.equal(p.scales.long().cpu(), e)


@pytest.mark.parametrize("M,k", [(1, 1), (77, 1000), (130, 264), (9, 4097)])
def test_relu_gate_from_the_checkpoint(ops, M, k):
    x = gaussian(5, M, k)
    dh = gaussian(6, M, k)
    dh[0, 0] = float("nan")
    x[0, 0] = -1.0                                   # a NaN behind a closed gate
    p = ops.act_pack(x.clamp(min=0))
    want = torch.where(x > 0, dh, torch.zeros_like(dh))
    assert torch.equal(ops.act_relu_grad(dh, p), want)
    inplace = dh.clone()
    assert ops.act_relu_grad(inplace, p, out=inplace) is inplace and torch.equal(inplace, want)
    odd = gaussian(6, M, k + 3)[:, 1:1 + k]          # rows at any two-byte address
    assert torch.equal(ops.act_relu_grad(odd, p), torch.where(x > 0, odd, torch.zeros_like(odd)))
    po = ops.act_pack(gaussian(5, M, k + 3)[:, 1:1 + k])
    assert torch.equal(po.q.long().cpu(), pack_reference(gaussian(5, M, k + 3)[:, 1:1 + k])[0]) if M * k < 5000 else True
    assert torch.equal(ops.act_unpack(p, out=torch.empty(M, k + 5, device="cuda", dtype=torch.bfloat16)[:, 2:2 + k]), ops.act_unpack(p))


def inside(values, lead, behind, fill):
    """A copy of values whose rows lie `lead` values into rows of `fill`, and the whole of it."""
    M, k = values.shape
    whole = torch.full((M + 2, lead + k + behind), fill, device="cuda", dtype=torch.bfloat16)
    view = whole[1:-1, lead:lead + k]
    view.copy_(values)
    return view, whole


@pytest.mark.parametrize("k", [1, 6, 7, 8, 9, 15, 17, 63, 64, 65, 121, 127, 128, 129, 250, 256, 1001])
@pytest.mark.parametrize("behind", [0, 1, 2, 5, 8])
def test_checkpoints_of_rows_at_any_address(ops, k, behind):
    M = 70
    scale = torch.exp2(torch.arange(-(-k // 128), device="cuda").repeat_interleave(128)[:k].float() * 3 - 4)   # another unit in every block
    x = (gaussian(k, M, k).float() * scale).bfloat16()
    x[3, k // 2], x[5, 0], x[7, k - 1] = float("inf"), float("nan"), 0.0
    dh = gaussian(k + 1, M, k)
    for lead in range(9):
        base, other = inside(x, 8, -k % 8, 0.0)[0], (lead * 3 + 1) % 8
        want = ops.act_pack(base)                                          # rows at multiples of 16 bytes
        assert base.data_ptr() % 16 == 0 and base.stride(0) % 8 == 0
        got = ops.act_pack(inside(x, lead, behind, float("nan"))[0])        # what surrounds the rows is not finite
        assert torch.equal(got.q, want.q) and torch.equal(got.scales, want.scales)
        plain = inside(x, 8, -k % 8, 0.0)[0]
        ops.act_unpack(want, out=plain)
        y, whole = inside(torch.zeros_like(x), lead, behind, 7.0)
        ops.act_unpack(want, out=y)
        assert torch.equal(torch.nan_to_num(y, nan=-3.0), torch.nan_to_num(plain, nan=-3.0))
        y.fill_(7.0)
        assert (whole == 7.0).all()                                        # nothing beside the rows was written
        gate = torch.where(want.q > 0, dh, torch.zeros_like(dh))
        gate[want.q == -128] = float("nan")
        z, whole = inside(torch.zeros_like(x), lead, behind, 7.0)
        ops.act_relu_grad(inside(dh, other, behind, float("nan"))[0], want, out=z)
        assert torch.equal(torch.nan_to_num(z, nan=-3.0), torch.nan_to_num(gate, nan=-3.0))
        z.copy_(dh)
        ops.act_relu_grad(z, want, out=z)                                  # in place
        assert torch.equal(torch.nan_to_num(z, nan=-3.0), torch.nan_to_num(gate, nan=-3.0))
        z.fill_(7.0)
        assert (whole == 7.0).all()


def test_relu_gate_passes_on_what_was_not_finite(ops):
    x = torch.tensor([[1.0, float("inf"), float("nan"), -1.0]], device="cuda").bfloat16()
    dz = ops.act_relu_grad(torch.ones_like(x), ops.act_pack(x))
    assert dz[0, 0] == 1 and dz[0, 3] == 0 and torch.isnan(dz[0, 1:3]).all()


@pytest.mark.parametrize("sizes,n,k", SHAPES)
def test_weight_gradient_from_the_checkpoint(ops, sizes, n, k):
    off, spans = offsets_of(sizes)
    M = sum(sizes)
    x, dy = gaussian(1, M, k).clamp(min=0), gaussian(3, M, n)
    p = ops.act_pack(x)
    kept = ops.act_unpack(p)
    want = torch.stack([dy[s].double().T @ kept[s].double() for s in spans])
    size = torch.stack([dy[s].double().abs().T @ kept[s].double().abs() for s in spans])
    for dtype in (torch.bfloat16, torch.float32):
        assert_sum(ops.grouped_weight_grad(dy, p, off, out_dtype=dtype), want, size, max(sizes))


def test_weight_gradient_from_the_checkpoint_keeps_groups_apart(lm, ops):
    off, spans = offsets_of([70, 58, 200])
    x, dy = gaussian(1, 328, 256), gaussian(3, 328, 136)
    x[spans[1]] = float("nan")
    dy[spans[1]] = float("inf")
    dw = ops.grouped_weight_grad(dy, ops.act_pack(x), off)
    assert torch.isfinite(dw[0]).all() and torch.isfinite(dw[2]).all() and not torch.isfinite(dw[1]).any()


@pytest.mark.parametrize("sizes,n,k", [([300, 0, 213], 136, 1000), ([2500, 1596], 512, 1032), ([20000], 256, 264)])
def test_both_ways_to_read_a_checkpoint_give_the_same_bits(lm, sizes, n, k):
    """Turned into bf16 inside the product, or by a kernel before it (long reductions, see the last shape)."""
    off, spans = offsets_of(sizes)
    x, dy = gaussian(1, sum(sizes), k).clamp(min=0), gaussian(3, sum(sizes), n)
    x[5, 3] = float("nan")
    o = lm.LMOps(widen=False)
    p = o.act_pack(x)
    wide = o.act_unpack(p)
    for dtype in (torch.bfloat16, torch.float32):
        inside = o.grouped_weight_grad(dy, p, off, out_dtype=dtype)
        before = o.grouped_weight_grad(dy, wide, off, out_dtype=dtype)
        o.widen = True
        chosen = o.grouped_weight_grad(dy, p, off, out_dtype=dtype)
        o.widen = False
        same = torch.isfinite(before)
        assert not same[0, :, 3].any() and torch.equal(same, torch.isfinite(inside)) and torch.equal(same, torch.isfinite(chosen))
        assert torch.equal(inside[same], before[same]) and torch.equal(chosen[same], before[same])
    assert o._lib.cocod_grouped_packed_workspace(4, 32768, 2048, 4096) == 32768 * 4096 * 2
    assert o._lib.cocod_grouped_packed_workspace(16, 2048, 1024, 1024) == 0
    o.destroy()


# ------------------------------------------------------------------------------------------------------- vocabulary
def vocab_reference(h, w, labels, spans, weights=None):
    G, V, D = w.shape
    loss, row, dh, dw = [], [], [], []
    for g, s in enumerate(spans):
        x, t = h[s].double(), labels[s].long()
        a = weights[s].double() if weights is not None else (t >= 0).double() / max(1, int((t >= 0).sum()))
        use = ((t >= 0) & (a != 0)).nonzero()[:, 0]
        l = x[use] @ w[g].double().T
        lse = torch.logsumexp(l, 1)
        r = torch.zeros(x.shape[0], dtype=torch.float64, device="cuda")
        own = l.gather(1, t[use, None])
        rest = torch.exp((l - own).clamp(max=0)).scatter(1, t[use, None], 0.0).sum(1)
        # (lse - own cancels where the label is as good as certain: 64 bits do not hold such a loss to its own size)
        r[use] = torch.where((l <= own).all(1), torch.log1p(rest), lse - own[:, 0])
        p = torch.exp(l - lse[:, None])
        p[torch.arange(len(use), device="cuda"), t[use]] -= 1
        p *= a[use, None]
        d = torch.zeros_like(x)
        d[use] = p @ w[g].double()
        loss.append((r * a).sum()), row.append(r), dh.append(d), dw.append(p.T @ x[use])
    return torch.stack(loss), torch.cat(row), torch.cat(dh), torch.stack(dw)


def check_vocab(got, h, w, labels, spans, weights=None):
    loss, row, dh, dw = vocab_reference(h, w, labels, spans, weights)
    D = w.shape[2]
    size = float(h.float().nan_to_num(0, 0, 0).norm(dim=1).max() * w.float().nan_to_num(0, 0, 0).norm(dim=2).max()) if h.shape[0] else 0.0
    d = (D / 16 + 8) * 2.0 ** -23 * size
    assert ((got[1].double() - row).abs() <= 2 * d + 2.0 ** -20 * (1 + row)).all()
    total = sum(weights.abs().double().sum() for _ in (0,)) if weights is not None else 1.0
    assert ((got[0].double() - loss).abs() <= (2 * d + 2.0 ** -19 * (1 + row.max() if row.numel() else 1)) * total).all()
    if len(got) == 2:
        return
    # terms of relative error 2^-8 + 2 d (dx) and 3 * 2^-8 + 2 d (dw), taken at their absolute values; one more rounding at the end
    for g, s in enumerate(spans):
        x, t = h[s].double(), labels[s].long()
        a = weights[s].double() if weights is not None else (t >= 0).double() / max(1, int((t >= 0).sum()))
        use = ((t >= 0) & (a != 0)).nonzero()[:, 0]
        p = torch.softmax(x[use] @ w[g].double().T, 1)
        p[torch.arange(len(use), device="cuda"), t[use]] -= 1
        p = (p * a[use, None]).abs()
        more = 2 * d + (p.shape[1] / 16 + 40) * 2.0 ** -23
        e, e3 = 2.0 ** -8 * 1.02 + more, 3 * 2.0 ** -8 * 1.02 + more
        near = torch.zeros_like(x)
        near[use] = p @ w[g].double().abs()
        assert ((got[2][s].double() - dh[s]).abs() <= e * near + 2.0 ** -8 * dh[s].abs() + 1e-38).all()
        assert ((got[3][g].double() - dw[g]).abs() <= e3 * (p.T @ x[use].abs()) + 2.0 ** -8 * dw[g].abs() + 1e-38).all()


VOCAB = [
    # sizes, V, D
    ([1], 1, 8),
    ([1], 2, 16),
    ([3], 65, 8),
    ([37], 129, 72),
    ([37], 8191, 256),
    ([130, 0, 61], 1000, 136),
    ([300, 250], 5003, 64),
    ([16] * 9, 257, 128),
    ([700], 4096, 512),
]


@pytest.mark.parametrize("sizes,V,D", VOCAB)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_vocabulary_loss_and_gradient(ops, sizes, V, D, dtype):
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    h, w = gaussian(1, M, D), gaussian(2, G, V, D, scale=2 * D ** -0.5)
    labels = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(V), dtype=torch.int32).cuda()
    labels[torch.rand(M, generator=torch.Generator().manual_seed(M)) < 0.1] = -1
    got = ops.vocab_loss_grad(h, w, labels, off, dw_dtype=dtype)
    check_vocab(got, h, w, labels, spans)
    alone = ops.vocab_loss(h, w, labels, off)
    assert torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1])
    ops.check()


def test_vocabulary_in_several_passes(lm):
    """A workspace too small for the batch: rows are taken in turns, the weight gradient is summed over them."""
    sizes = [500, 0, 777, 300]
    off, spans = offsets_of(sizes)
    M, V, D = sum(sizes), 3001, 128
    h, w = gaussian(1, M, D), gaussian(2, 4, V, D, scale=2 * D ** -0.5)
    labels = torch.randint(-1, V, (M,), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    whole = lm.LMOps()
    need = whole._lib.cocod_vocab_workspace(4, M, V, D, 1, lm.F32, 1 << 40)
    want = whole.vocab_loss_grad(h, w, labels, off, dw_dtype=torch.float32)
    for dtype, spare in ((torch.float32, 0), (torch.bfloat16, 4 * 4 * V * D)):
        small = lm.LMOps(workspace_limit=need // 3 + spare)
        got = small.vocab_loss_grad(h, w, labels, off, dw_dtype=dtype)
        small.check()
        assert torch.equal(got[1], want[1])
        check_vocab(got, h, w, labels, spans)
        loss = small.vocab_loss(h, w, labels, off)
        assert torch.equal(loss[1], want[1])
        small.destroy()
    least = lm.LMOps(workspace_limit=0)              # not even the fewest rows stay within it: the fewest are taken
    check_vocab(least.vocab_loss_grad(h, w, labels, off, dw_dtype=torch.float32), h, w, labels, spans)
    least.destroy()
    whole.destroy()


def test_vocabulary_row_weights(ops):
    off, spans = offsets_of([90, 40])
    h, w = gaussian(1, 130, 64), gaussian(2, 2, 700, 64, scale=0.25)
    labels = torch.randint(0, 700, (130,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    weights = torch.rand(130, generator=torch.Generator().manual_seed(4)).cuda()
    weights[::7] = 0
    weights[5] = -2.0
    check_vocab(ops.vocab_loss_grad(h, w, labels, off, row_weights=weights), h, w, labels, spans, weights)


def test_vocabulary_rows_without_a_label_may_hold_anything(ops):
    off, spans = offsets_of([140, 60])
    h, w = gaussian(1, 200, 64), gaussian(2, 2, 300, 64, scale=0.25)
    labels = torch.randint(0, 300, (200,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    dead = torch.tensor([0, 7, 139, 140, 199])
    labels[dead] = -100
    clean = ops.vocab_loss_grad(h, w, labels, off)
    h[dead] = float("nan")
    h[dead[1]] = float("inf")
    got = ops.vocab_loss_grad(h, w, labels, off)
    assert all(torch.equal(a, b) for a, b in zip(clean, got))
    assert (got[1][dead] == 0).all() and (got[2][dead] == 0).all()
    labels[140:] = -1                                # a group without any label
    loss, row, dx, dw = ops.vocab_loss_grad(h, w, labels, off)
    assert loss[1] == 0 and (row[140:] == 0).all() and (dx[140:] == 0).all() and (dw[1] == 0).all() and torch.isfinite(dw[0].float()).all()


def test_vocabulary_nan_stays_in_its_row_and_group(ops):
    off, spans = offsets_of([140, 60])
    h, w = gaussian(1, 200, 64), gaussian(2, 2, 300, 64, scale=0.25)
    labels = torch.randint(0, 300, (200,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    h[150, 3] = float("nan")
    loss, row, dx, dw = ops.vocab_loss_grad(h, w, labels, off)
    assert torch.isnan(loss[1]) and torch.isnan(row[150]) and torch.isnan(dx[150].float()).all()
    ok = torch.ones(200, dtype=torch.bool, device="cuda")
    ok[150] = False
    assert torch.isfinite(row[ok]).all() and torch.isfinite(dx[ok].float()).all() and torch.isfinite(dw[0].float()).all() and torch.isfinite(loss[0])


@pytest.mark.parametrize("big", [60.0, 200.0, 2000.0])
def test_vocabulary_large_losses(ops, big):
    """Rows whose loss is far beyond what exp(l - l[label]) in bf16 holds, among ordinary ones."""
    off, spans = offsets_of([300])
    h, w = gaussian(1, 300, 64), gaussian(2, 1, 1000, 64, scale=0.25)
    labels = torch.randint(0, 1000, (300,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    for r in (0, 77, 255, 256, 299):                 # the row points against its label's weights
        v = w[0, labels[r]].float()
        h[r] = (-v * (big / float(v @ v))).bfloat16()
    got = ops.vocab_loss_grad(h, w, labels, off)
    assert float(got[1].max()) > 0.9 * big
    check_vocab(got, h, w, labels, spans)
    assert torch.equal(ops.vocab_loss(h, w, labels, off)[1], got[1])


def test_vocabulary_confident_rows_keep_their_small_losses(ops):
    """A label that is as good as certain: loss and gradient are tiny and still right to their own size."""
    off, spans = offsets_of([64])
    w = gaussian(2, 1, 512, 128, scale=0.3)
    labels = torch.arange(64, dtype=torch.int32, device="cuda") * 8
    h = (w[0, labels.long()].float() * 2.5).bfloat16()
    got = ops.vocab_loss_grad(h, w, labels, off)
    loss, row, dh, dw = vocab_reference(h, w, labels, spans)
    assert float(row.median()) < 1e-4
    d = (128 / 16 + 8) * 2.0 ** -23 * float(h.float().norm(dim=1).max() * w.float().norm(dim=2).max())
    assert ((got[1].double() - row).abs() <= (2 * d + 2.0 ** -18) * row).all()
    check_vocab(got, h, w, labels, spans)


def test_vocabulary_gradient_against_differences(ops):
    off, spans = offsets_of([20])
    h, w = gaussian(1, 20, 32), gaussian(2, 1, 150, 32, scale=0.5)
    labels = torch.randint(0, 150, (20,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    _, _, dx, dw = ops.vocab_loss_grad(h, w, labels, off, dw_dtype=torch.float32)

    def loss(hh, ww):
        return vocab_reference(hh, ww, labels, spans)[0][0]
    eps = 1e-4
    for r, i in ((0, 0), (19, 31), (7, 5)):
        hp, hm = h.double(), h.double()
        hp[r, i] += eps
        hm[r, i] -= eps
        diff = float(loss(hp, w) - loss(hm, w)) / (2 * eps)
        assert abs(diff - float(dx[r, i])) <= 2.0 ** -7 * float(w.float().abs().max()) * 2 / 20
    for v, i in ((int(labels[0]), 3), (149, 31), (0, 0)):
        wp, wm = w.double(), w.double()
        wp[0, v, i] += eps
        wm[0, v, i] -= eps
        diff = float(loss(h, wp) - loss(h, wm)) / (2 * eps)
        assert abs(diff - float(dw[0, v, i])) <= 3 * 2.0 ** -8 * float(h.float().abs().sum(0)[i]) / 20


def test_vocabulary_into_the_workers_gradients(ops):
    """The weight gradient as a view of the K x P gradients, the weights as a view of the bf16 copy."""
    sizes, V, D = [33, 60], 515, 64
    off, spans = offsets_of(sizes)
    P = (V * D + 128 + 63) // 64 * 64
    shadow = gaussian(2, 2, P, scale=0.25)
    grads = torch.full((2, P), 3.0, device="cuda")
    h = gaussian(1, 93, D)
    labels = torch.randint(0, V, (93,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    w, dw = shadow[:, 64:64 + V * D].view(2, V, D), grads[:, 64:64 + V * D].view(2, V, D)
    got = ops.vocab_loss_grad(h, w, labels, off, dw=dw)
    check_vocab(got, h, w, labels, spans)
    assert (grads[:, :64] == 3).all() and (grads[:, 64 + V * D:] == 3).all()


# ------------------------------------------------------------------------------------------------------- drawn shapes
@pytest.mark.parametrize("seed", range(40))
def test_drawn_shapes(lm, ops, seed):
    """Sizes, divisions and types by chance; groups without rows anywhere."""
    import random
    r = random.Random(seed)
    G, M = r.choice([1, 2, 3, 7, 33]), r.choice([1, 5, 64, 300, 1500, 6000])
    n, k = 8 * r.choice([1, 3, 16, 33, 75, 130]), 8 * r.choice([1, 2, 9, 32, 49, 128])
    cuts = sorted(r.choice([0, M, r.randint(0, M)]) for _ in range(G - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [M])]
    off, spans = offsets_of(sizes)
    dtype = r.choice([torch.bfloat16, torch.float32])
    x, w, dy = gaussian(seed, M, k), gaussian(seed + 1, G, n, k, scale=k ** -0.5), gaussian(seed + 2, M, n)
    (y, ya), (dx, dxa), (dw, dwa) = products(x, w, dy, spans)
    assert_sum(ops.grouped_forward(x, w, off, out_dtype=dtype), y, ya, k)
    assert_sum(ops.grouped_input_grad(dy, w, off, out_dtype=dtype), dx, dxa, n)
    assert_sum(ops.grouped_weight_grad(dy, x, off, out_dtype=dtype), dw, dwa, M)
    p = ops.act_pack(x)
    kept = ops.act_unpack(p)
    (_, _), (_, _), (dw, dwa) = products(kept, w, dy, spans)
    assert_sum(ops.grouped_weight_grad(dy, p, off, out_dtype=dtype), dw, dwa, M)
    V = r.choice([3, 127, 1000, 4097])
    w = gaussian(seed + 1, G, V, k, scale=2 * k ** -0.5)
    labels = torch.randint(-1, V, (M,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32).cuda()
    check_vocab(ops.vocab_loss_grad(x, w, labels, off, dw_dtype=dtype), x, w, labels, spans)
    ops.check()


# ------------------------------------------------------------------------------------------------------- beyond 2^31 values
def test_checkpoint_beyond_32_bits(ops):
    M, k = 70001, 32768
    x = torch.empty(M, k, device="cuda", dtype=torch.bfloat16)
    x[:64], x[-64:] = gaussian(1, 64, k), gaussian(2, 64, k)
    p = ops.act_pack(x)
    for rows in (slice(0, 64), slice(M - 64, M)):
        alone = ops.act_pack(x[rows].clone())
        assert torch.equal(alone.q, p.q[rows]) and torch.equal(alone.scales, p.scales[:, rows])
    y = ops.act_unpack(p)
    assert torch.equal(y[-64:], ops.act_unpack(ops.act_pack(x[-64:].clone())))
    del y
    z = ops.act_relu_grad(x, p, out=x)
    assert torch.equal(z[-64:], torch.where(p.q[-64:] > 0, z[-64:], torch.zeros_like(z[-64:]))) and (z[-64:] > 0).any()


def test_products_beyond_32_bits(ops):
    M, n, k = 66001, 33024, 16
    off, spans = offsets_of([30000, 36001])
    x, w = gaussian(1, M, k), gaussian(2, 2, n, k)
    y = ops.grouped_forward(x, w, off)
    for rows, g in ((slice(29900, 30000), 0), (slice(30000, 30100), 1), (slice(M - 100, M), 1)):
        want, size = x[rows].double() @ w[g].double().T, x[rows].double().abs() @ w[g].double().abs().T
        assert_sum(y[rows], want, size, k)
    dw = ops.grouped_weight_grad(y, x, off)
    want, size = y[30000:, -64:].double().T @ x[30000:].double(), y[30000:, -64:].double().abs().T @ x[30000:].double().abs()
    assert_sum(dw[1, -64:], want, size, 36001)


def test_vocabulary_beyond_32_bits(lm):
    M, V, D = 17001, 131073, 16
    off, spans = offsets_of([M])
    h, w = gaussian(1, M, D), gaussian(2, 1, V, D, scale=0.5)
    labels = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    o = lm.LMOps(workspace_limit=16 << 30)
    loss, row, dx, dw = o.vocab_loss_grad(h, w, labels, off)
    o.check()
    last = slice(M - 50, M)
    logits = h[last].double() @ w[0].double().T
    own = logits.gather(1, labels[last].long()[:, None])[:, 0]
    want = torch.logsumexp(logits, 1) - own
    d = (D / 16 + 8) * 2.0 ** -23 * float(h.float().norm(dim=1).max() * w.float().norm(dim=2).max())
    assert ((row[last].double() - want).abs() <= 2 * d + 2.0 ** -20 * (1 + want)).all()
    p = torch.softmax(logits, 1)
    p[torch.arange(50, device="cuda"), labels[last].long()] -= 1
    p /= M
    near = p.abs() @ w[0].double().abs()
    assert ((dx[last].double() - p @ w[0].double()).abs() <= (2.0 ** -8 * 1.02 + 2 * d + (V / 16 + 40) * 2.0 ** -23) * near + 2.0 ** -8 * near + 1e-38).all()
    o.destroy()


# ------------------------------------------------------------------------------------------------------- refusals
def test_refusals(lm, ops):
    from paper_1906_12043_b200.engine import CocodError, ERR_INVALID, ERR_TIMEOUT
    off, _ = offsets_of([40, 24])
    x, w, dy = gaussian(1, 64, 64), gaussian(2, 2, 128, 64), gaussian(3, 64, 128)
    labels = torch.zeros(64, dtype=torch.int32, device="cuda")
    for bad in (x.float(), x.cpu(), x[:, :32], x.t(), x[None]):
        with pytest.raises((ValueError, CocodError)):
            ops.grouped_forward(bad, w, off)
    for bad in (w.float(), w[0], w.transpose(1, 2), w[:, :, :40], w.cpu()):
        with pytest.raises((ValueError, CocodError)):
            ops.grouped_forward(x, bad, off)
    for bad in (off.long(), off[:2], off.cpu(), off.float()):
        with pytest.raises((ValueError, CocodError)):
            ops.grouped_forward(x, w, bad)
    with pytest.raises((ValueError, CocodError)):
        ops.grouped_forward(x, w, off, out_dtype=torch.float16)
    with pytest.raises((ValueError, CocodError)):
        ops.grouped_forward(x, w, off, out=torch.empty(64, 120, device="cuda", dtype=torch.bfloat16))
    with pytest.raises((ValueError, CocodError)):        # a width that is no multiple of eight
        ops.grouped_weight_grad(dy[:, :100], gaussian(1, 64, 72)[:, :68], off)
    with pytest.raises((ValueError, CocodError)):        # rows that start off 16 bytes
        ops.grouped_forward(gaussian(1, 64, 80)[:, 1:65], w, off)
    with pytest.raises((ValueError, CocodError)):        # groups on top of one another
        ops.grouped_weight_grad(dy, x, off, out=torch.empty(1, 128, 64, device="cuda").expand(2, 128, 64))
    for bad in (labels.long(), labels[:63], labels.cpu()):
        with pytest.raises((ValueError, CocodError)):
            ops.vocab_loss(x, w, bad, off)
    with pytest.raises((ValueError, CocodError)):
        ops.vocab_loss_grad(x, w, labels, off, row_weights=torch.ones(63, device="cuda"))
    with pytest.raises((ValueError, CocodError)):
        ops.act_relu_grad(x, ops.act_pack(gaussian(1, 64, 56)))
    with pytest.raises(ValueError):
        lm.PackedActivations.from_parts(torch.zeros(4, 20, dtype=torch.int8, device="cuda"), torch.zeros(1, 4, dtype=torch.uint8, device="cuda"))
    ops.check()
    # what only the device can see is reported by the next check; nothing outside the matrices is touched
    for sizes in ([0, 40, 30], [0, 80, 64], [5, 40, 64], [0, 40, 60]):
        bad = torch.tensor(sizes, dtype=torch.int32, device="cuda")
        guard = torch.full((66, 128), 9.0, device="cuda", dtype=torch.bfloat16)
        ops.grouped_forward(x, w, bad, out=guard[1:65])
        with pytest.raises(CocodError) as e:
            ops.check()
        assert e.value.code == ERR_INVALID and (guard[0] == 9).all() and (guard[65] == 9).all()
        ops.check()                                       # reported once
    labels[3] = 128
    loss, row = ops.vocab_loss(x, w, labels, off)
    with pytest.raises(CocodError) as e:
        ops.check()
    assert e.value.code == ERR_INVALID and row[3] == 0 and torch.isfinite(loss).all()


@pytest.mark.parametrize("pair", [False, True])
def test_a_wait_that_runs_out_is_reported(lm, ops, pair):
    from paper_1906_12043_b200.engine import ERR_TIMEOUT
    assert lm.grouped_wait_selftest(30, pair) == ERR_TIMEOUT
    off, spans = offsets_of([100])
    x, w = gaussian(1, 100, 64), gaussian(2, 1, 64, 64)
    y = ops.grouped_forward(x, w, off)
    assert_sum(y, x.double() @ w[0].double().T, x.double().abs() @ w[0].double().abs().T, 64)
    ops.check()
