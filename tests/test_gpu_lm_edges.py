"""The language-model operators where they are easily wrong: what lies beside a checkpoint, very long and very wide products, the
vocabulary's largest term, streams and repeated calls.

Tolerances are derived beside each test.
"""
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


def half_unit(x):
    """Half a unit in the last place of bf16 (8 significant bits) at the values x."""
    return torch.exp2(torch.frexp(x)[1].double() - 9)


# ------------------------------------------------------------------------------------------------------- vocabulary
@pytest.mark.parametrize("sizes,V,D", [([37], 8191, 256), ([300, 0, 77], 1000, 264), ([1], 50, 8)])
def test_the_label_s_term_of_dx_is_rounded_once(ops, sizes, V, D):
    """All rows have the same label, whose row of w is the only one that is not 0, so that dx is that one term, a (softmax - 1) w: its sum is in
    fp32 and the result rounds it once.  A logit is off by at most (D / 16 + 8) * 2^-23 |h| |w| < 2^-13 for |h| |w| <= 2^5 here, and the
    term by no more than that much of itself (d (1 - softmax) / (1 - softmax) = softmax)."""
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    h = gaussian(1, M, D)
    w = torch.zeros(G, V, D, device="cuda", dtype=torch.bfloat16)
    w[:, V // 3] = gaussian(2, G, D, scale=D ** -0.5)
    labels = torch.full((M,), V // 3, dtype=torch.int32, device="cuda")
    assert float(h.float().norm(dim=1).max() * w.float().norm(dim=2).max()) <= 32
    for dtype in (torch.bfloat16, torch.float32):
        dx = ops.vocab_loss_grad(h, w, labels, off, dw_dtype=dtype)[2].double()
        for g, s in enumerate(spans):
            l = h[s].double() @ w[g].double().T
            want = ((torch.softmax(l, 1)[:, V // 3] - 1) / max(1, sizes[g]))[:, None] * w[g, V // 3].double()
            assert ((dx[s] - want).abs() <= half_unit(want) + 2.0 ** -13 * want.abs()).all()
    ops.check()


# ------------------------------------------------------------------------------------------------------- checkpoints
@pytest.mark.parametrize("M,k", [(1, 1), (1, 7), (1, 1001), (3, 9), (33, 100), (70, 129), (40, 263), (5, 520)])
def test_a_checkpoint_in_a_view_leaves_its_surroundings(lm, ops, M, k):
    """q as columns of a wider buffer, and one that ends with its last value and has its scales right behind: neither is written nor used
    beyond the k values of a row, and what is read from it is what an own checkpoint gives."""
    x = gaussian(1, M, k)
    own = ops.act_pack(x)
    wide = torch.full((M, -(-k // 16) * 16 + 32), 77, device="cuda", dtype=torch.int8)
    blocks = -(-k // 128)
    at = (M - 1) * (-(-k // 16) * 16) + k
    flat = torch.full((at + blocks * M + 64,), 77, device="cuda", dtype=torch.int8)
    views = [(wide[:, 16:16 + k], torch.full((blocks, M), 77, device="cuda", dtype=torch.uint8)),
             (torch.as_strided(flat, (M, k), (-(-k // 16) * 16, 1)), flat[at:at + blocks * M].view(torch.uint8).view(blocks, M))]
    dh = gaussian(2, M, k + 1)
    for q, scales in views:
        p = lm.PackedActivations.from_parts(q, scales)
        for _ in range(3):
            assert ops.act_pack(x, out=p) is p
            assert torch.equal(q, own.q) and torch.equal(scales, own.scales)
        assert torch.equal(ops.act_unpack(p), ops.act_unpack(own))
        for d in (dh[:, :k], dh[:, 1:]):
            assert torch.equal(ops.act_relu_grad(d, p), ops.act_relu_grad(d, own))
            other = torch.empty(M, k + 1, device="cuda", dtype=torch.bfloat16)[:, 1:]
            assert torch.equal(ops.act_relu_grad(d, p, out=other), ops.act_relu_grad(d, own))
            assert torch.equal(ops.act_unpack(p, out=other), ops.act_unpack(own))
        if k % 8 == 0:
            off, _ = offsets_of([M])
            assert torch.equal(ops.grouped_weight_grad(gaussian(3, M, 16), p, off), ops.grouped_weight_grad(gaussian(3, M, 16), own, off))
    assert (wide[:, :16] == 77).all() and (wide[:, 16 + k:] == 77).all() and (flat[at + blocks * M:] == 77).all()
    gaps = torch.ones(at, dtype=torch.bool, device="cuda")
    torch.as_strided(gaps, (M, k), (-(-k // 16) * 16, 1)).fill_(False)
    assert (flat[:at][gaps] == 77).all()
    ops.check()


# ------------------------------------------------------------------------------------------------------- products
@pytest.mark.parametrize("rows", [1, 2])
def test_weight_gradient_of_few_rows_into_very_wide_ones(ops, rows):
    """8 x 2^25 results from one or two rows: as many tile columns as a band of 65536 tile rows would overflow 32 bits with.  Each result is at
    most two products of bf16, exact in fp32, and their sum, which the tensor cores cut off by at most 2^-22 of the products' magnitude."""
    n, k = 8, 1 << 25
    off, _ = offsets_of([rows])
    dy, x = gaussian(1, rows, n), gaussian(2, rows, k)
    dw = ops.grouped_weight_grad(dy, x, off, out=torch.full((1, n, k), 7.0, device="cuda"))
    ops.check()
    for at in range(0, k, 1 << 23):
        part = slice(at, at + (1 << 23))
        want = dy.double().T @ x[:, part].double()
        assert ((dw[0, :, part].double() - want).abs() <= 2.0 ** -22 * (dy.double().abs().T @ x[:, part].double().abs())).all()


# ------------------------------------------------------------------------------------------------------- vocabulary, second pass
def test_means_after_a_second_pass_hold_every_row(ops):
    """Losses above 50 in rows of every block of 32, so that the rows are done again and the blocks that end last add the losses up: the means are
    those of the losses that are returned (sums of n positive fp32 values in any order: within n * 2^-23 of themselves), every time."""
    sizes, V, D = [700, 0, 1500, 333], 300, 16
    off, spans = offsets_of(sizes)
    h, w = gaussian(1, sum(sizes), D), gaussian(2, len(sizes), V, D)
    h[::7] *= 40
    labels = torch.randint(0, V, (sum(sizes),), generator=torch.Generator().manual_seed(3)).int().cuda()
    first = ops.vocab_loss(h, w, labels, off)
    assert (first[1].view(-1)[::7] > 50).any()
    for _ in range(200):
        loss, row = ops.vocab_loss(h, w, labels, off)
        assert torch.equal(row, first[1]) and torch.equal(loss, first[0])
    for g, s in enumerate(spans):
        want = first[1][s].double().sum() / max(1, sizes[g])
        assert abs(float(first[0][g] - want)) <= 2.0 ** -23 * max(sizes) * float(want)
    ops.check()


@pytest.mark.parametrize("sizes,n,k", [([2500, 1596], 512, 1032), ([300, 0, 213, 4000], 1024, 520)])
def test_checkpoints_turned_inside_the_product_always_give_the_same_bits(lm, sizes, n, k):
    """Operand tiles that converting warps write, in single thread blocks and in pairs: every repetition gives what the checkpoint in bf16 gives."""
    o = lm.LMOps(widen=False)
    off, _ = offsets_of(sizes)
    x, dy = gaussian(1, sum(sizes), k).relu(), gaussian(2, sum(sizes), n)
    p = o.act_pack(x)
    for dtype in (torch.bfloat16, torch.float32):
        want = o.grouped_weight_grad(dy, o.act_unpack(p), off, out_dtype=dtype)
        for _ in range(150):
            assert torch.equal(o.grouped_weight_grad(dy, p, off, out_dtype=dtype), want)
    o.check()
    o.destroy()


# ------------------------------------------------------------------------------------------------------- streams
def test_a_report_outlives_the_creation_on_a_busy_stream(lm):
    """Operators made while the default stream is busy, and used at once on a stream of their own: what the first call reports stands."""
    from paper_1906_12043_b200.engine import CocodError, ERR_INVALID
    x, w = gaussian(1, 64, 64), gaussian(2, 2, 64, 64)
    bad = torch.tensor([0, 40, 30], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    lm.LMOps().grouped_forward(x, w, bad)
    torch.cuda.synchronize()
    torch.cuda._sleep(400_000_000)                         # about 0.2 s
    o = lm.LMOps()
    with torch.cuda.stream(side):
        o.grouped_forward(x, w, bad)
    torch.cuda.synchronize()
    with torch.cuda.stream(side), pytest.raises(CocodError) as e:
        o.check()
    assert e.value.code == ERR_INVALID
    o.check()
    o.destroy()


def test_long_sums_of_positive_products_do_not_shrink(ops):
    """bf16 results of 2^19 positive products each, in tiles that are not cut.  The tensor cores add in parts of 32768 products: each of a part's
    2048 steps cuts off at most a unit in the last place of the running sum, 2^-23 of it, and that is half of the part's on average, so
    that a result is too small by at most 2^-13 of itself.  The mean over 4096 results shows it: their roundings (at most 2^-8, of
    either sign) leave 5 * 2^-8 / sqrt(12) / 64 < 2^-13 of it."""
    M, n, k = 2304, 2304, 1 << 19
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w = ((torch.rand(M, k, generator=g, device="cuda") + 0.5).bfloat16() for _ in range(2))
    y = ops.grouped_forward(x, w[None], torch.tensor([0, M], dtype=torch.int32, device="cuda"))
    ops.check()
    want = x[:64].double() @ w[:64].double().T
    assert abs(float((y[:64, :64].double() / want - 1).mean())) <= 2.0 ** -12


@pytest.mark.parametrize("n,k", [(24, 40), (136, 264), (1024, 1032)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("few", [True, False])
def test_every_remainder_of_a_group_beside_rows_that_are_not_finite(lm, n, k, packed, few):
    """Groups of every length modulo 64, each followed by one whose rows are NaN and infinite: nothing of those comes in, and they are NaN.
    fp32 results of up to 200 products: 13 steps that cut off at most 2^-23 of the sum of magnitudes, and as much again for the joining of parts."""
    lengths = [1, 15, 16, 17, 31, 47, 48, 49, 63, 64, 65, 127, 129, 177, 200] if few else list(range(1, 66)) + [100, 190]
    sizes = [s for length in lengths for s in (length, 1 + length % 5)][:32 if few else None]
    off, spans = offsets_of(sizes)
    M, G = sum(sizes), len(sizes)
    assert (G > 32) != few
    x, dy = gaussian(1, M, k), gaussian(2, M, n)
    for s in spans[1::2]:
        x[s], dy[s] = float("nan"), float("inf")
    o = lm.LMOps(widen=False)
    a = o.act_pack(x) if packed else x
    if packed:
        x = o.act_unpack(a)
    for dtype in (torch.float32, torch.bfloat16):
        dw = o.grouped_weight_grad(dy, a, off, out_dtype=dtype)
        for g, s in enumerate(spans):
            if g % 2:
                assert torch.isnan(dw[g]).all()
                continue
            want, size = dy[s].double().T @ x[s].double(), dy[s].double().abs().T @ x[s].double().abs()
            bound = 26 * 2.0 ** -23 * size + (half_unit(want) * 1.01 if dtype == torch.bfloat16 else 0)
            assert ((dw[g].double() - want).abs() <= bound).all()
    o.check()
    o.destroy()


# ------------------------------------------------------------------------------------------------------- beyond 2^31 values
def test_open_gates_beyond_32_bits_pass_their_values(ops):
    M, k = 70001, 32768
    x = torch.empty(M, k, device="cuda", dtype=torch.bfloat16)
    ends = [slice(0, 64), slice(M - 64, M)]
    for i, rows in enumerate(ends):
        x[rows] = gaussian(i, 64, k)
    p = ops.act_pack(x)
    for i, rows in enumerate(ends):
        x[rows] = gaussian(i + 2, 64, k)
    ops.act_relu_grad(x, p, out=x)
    for i, rows in enumerate(ends):
        assert torch.equal(x[rows], torch.where(gaussian(i, 64, k) > 0, gaussian(i + 2, 64, k), 0.0).bfloat16())
    ops.check()


def test_gradient_of_the_weights_beyond_32_bits(lm):
    """dw of both ends of a vocabulary, over more than 2^31 exponentials.  A term carries three bf16 roundings (3 * 2^-8) and twice a logit's
    error d (each step of 16 products cuts off at most 2^-23 of |h| |w|), the result one more; the sum of M terms M / 16 + 40 steps."""
    M, V, D = 17001, 131073, 16
    off, _ = offsets_of([M])
    h, w = gaussian(1, M, D), gaussian(2, 1, V, D, scale=0.5)
    labels = torch.randint(0, V, (M,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    labels[::9] = V - 3
    o = lm.LMOps(workspace_limit=16 << 30)
    dw = o.vocab_loss_grad(h, w, labels, off)[3][0].double()
    o.check()
    o.destroy()
    lse = torch.cat([torch.logsumexp(part.double() @ w[0].double().T, 1) for part in h.split(1000)])
    d = (D / 16 + 8) * 2.0 ** -23 * float(h.float().norm(dim=1).max() * w.float().norm(dim=2).max())
    for at in (slice(0, 40), slice(V - 40, V)):
        p = torch.exp(h.double() @ w[0, at].double().T - lse[:, None])
        p -= (labels.long()[:, None] == torch.arange(V, device="cuda")[None, at]).double()
        want, size = p.T @ h.double() / M, p.abs().T @ h.double().abs() / M
        assert ((dw[at] - want).abs() <= (3 * 2.0 ** -8 * 1.02 + 2 * d + (M / 16 + 40) * 2.0 ** -23) * size + 2.0 ** -8 * want.abs()).all()


# ------------------------------------------------------------------------------------------------------- refusals
def test_a_call_while_another_device_is_current_is_refused_by_name(lm):
    """(As if the operators had been made on the next device, which need not exist.)"""
    o = lm.LMOps()
    here, other = torch.cuda.current_device(), torch.cuda.current_device() + 1
    x, w, off = gaussian(1, 64, 64), gaussian(2, 1, 64, 64), torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    labels, p = torch.zeros(64, dtype=torch.int32, device="cuda"), o.act_pack(x)
    o._device = other
    o._here = lambda packed: None
    for call in (lambda: o.grouped_forward(x, w, off), lambda: o.grouped_input_grad(x, w, off), lambda: o.grouped_weight_grad(x, x, off),
                 lambda: o.grouped_weight_grad(x, p, off), lambda: o.act_pack(x), lambda: o.act_pack(x, out=p), lambda: o.act_unpack(p),
                 lambda: o.act_relu_grad(x, p), lambda: o.vocab_loss(x, w, labels, off), lambda: o.vocab_loss_grad(x, w, labels, off)):
        with pytest.raises(ValueError, match=f"current device is cuda:{here}.*made on cuda:{other}"):
            call()
    o._device = here
    o.grouped_forward(x, w, off)
    o.check()
    o.destroy()


def test_no_room_for_a_result_is_torch_s_own_error(ops):
    dy, off = gaussian(1, 8, 1 << 19), torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        ops.grouped_weight_grad(dy, dy, off)               # 2^38 fp32 values
    assert torch.isfinite(ops.grouped_weight_grad(dy[:, :64], dy[:, :64], off)).all()
    ops.check()


def test_results_on_top_of_operands_are_refused(ops):
    x, w, off = gaussian(1, 64, 64), gaussian(2, 1, 64, 64), torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    labels = torch.zeros(64, dtype=torch.int32, device="cuda")
    two = gaussian(3, 128, 64)
    for call in (lambda: ops.grouped_forward(x, w, off, out=x), lambda: ops.grouped_forward(x, w, off, out=w[0]),
                 lambda: ops.grouped_forward(two[:64], w, off, out=two[1:65]), lambda: ops.grouped_input_grad(x, w, off, out=x),
                 lambda: ops.grouped_weight_grad(x, two[:64], off, out=x[None]), lambda: ops.grouped_weight_grad(two[:64], x, off, out=x[None]),
                 lambda: ops.grouped_weight_grad(x, ops.act_pack(x), off, out=x[None]), lambda: ops.act_relu_grad(two[:64], ops.act_pack(x), out=two[1:65]),
                 lambda: ops.vocab_loss_grad(x, w, labels, off, dw=w), lambda: ops.vocab_loss_grad(x, w, labels, off, dw=x[None])):
        with pytest.raises(ValueError, match="lies on"):
            call()
    # beside one another in one buffer, and in place where that is meant
    buffer = torch.cat([x, x], 1)
    assert torch.equal(ops.grouped_forward(buffer[:, :64], w, off, out=buffer[:, 64:]), ops.grouped_forward(x, w, off))
    want = ops.act_relu_grad(x, ops.act_pack(two[:64]))
    assert torch.equal(ops.act_relu_grad(x, ops.act_pack(two[:64]), out=x.view(64, 64)), want)
    ops.check()


@pytest.mark.parametrize("weight", [1e-25, -3e-20, 1e-3])
def test_small_weights_of_rows_with_large_losses(ops, weight):
    """Losses of 30 to 49, for which exp(loss) alone takes up half of fp32's range: dx and dw keep their size.  A term of dx is off by one bf16
    rounding and twice a logit's error d (each of D / 16 + 8 steps cuts off at most 2^-23 of |h| |w|), of dw by three; the result by one more,
    which is up to half of 2^-133, bf16's least unit, for results below 2^-126."""
    M, V, D = 40, 500, 64
    off, _ = offsets_of([M])
    h, w = gaussian(1, M, D), gaussian(2, 1, V, D, scale=D ** -0.5)
    labels = torch.randint(0, V - 1, (M,), generator=torch.Generator().manual_seed(3)).int().cuda()
    h = (h.float() * torch.linspace(28, 44, M, device="cuda")[:, None] / (h.float() @ w[0, -1].float())[:, None]).bfloat16()
    weights = torch.full((M,), weight, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        loss, row, dx, dw = ops.vocab_loss_grad(h, w, labels, off, row_weights=weights, dw_dtype=dtype)
        l = h.double() @ w[0].double().T
        want = torch.logsumexp(l, 1) - l.gather(1, labels.long()[:, None])[:, 0]
        assert float(want.max()) > 40
        d = (D / 16 + 8) * 2.0 ** -23 * float(h.float().norm(dim=1).max() * w.float().norm(dim=2).max())
        assert ((row.double() - want).abs() <= 2 * d + 2.0 ** -20 * (1 + want)).all()
        p = torch.softmax(l, 1)
        p[torch.arange(M, device="cuda"), labels.long()] -= 1
        p *= weights.double()[:, None]
        more = 2 * d + (V / 16 + 40) * 2.0 ** -23
        for got, to, size, terms in ((dx, p @ w[0].double(), p.abs() @ w[0].double().abs(), 1), (dw[0], p.T @ h.double(), p.abs().T @ h.double().abs(), 3)):
            assert ((got.double() - to).abs() <= (terms * 2.0 ** -8 * 1.02 + more) * size + 2.0 ** -8 * to.abs() + 2.0 ** -134).all()
    ops.check()
