"""AdamW over many tensors (optim.AdamW, optim.EngineAdamW) against the formulas in 64 bits.

Tolerances, derived before the first run.  With u = 2^-24:

* m: two products, a sum and two rounded constants: 3 u (beta1 |m| + (1 - beta1) |g|); v likewise with the square: 4 u v.
* p: p (1 - lr decay) carries 2 u; the update's factors: m (above, relative to its terms), the root 2 u + u, the correction 2 u, the sum 2 u, the quotient 2 ulp = 4 u, the rate
  2 u, so 16 u times (beta1 |m| + (1 - beta1) |g|) / denominator * rate, the last sum u |p|: 4 u |p| + 16 u * that.  A bf16 parameter adds 2^-8 of the value.
* 8 bits: the definition names every rounding between the old moments and the new ones, so that codes and units are equal to those of the formulas in fp32, one
  correctly rounded operation after the other (done here in 64 bits, rounded to 32 after each: for sums, products, quotients and roots of fp32 that is the correct rounding).
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EMPTY = 2.0 ** -100


@pytest.fixture(scope="module")
def optim():
    from paper_1906_12043_b200 import build, optim
    build.build()
    return optim


def gaussian(seed, *shape, scale=1.0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def f32(x):
    return x.float().double()


def padded(t):
    out = torch.zeros(-(-t.numel() // 128) * 128, dtype=t.dtype, device="cuda")
    out[:t.numel()] = t.reshape(-1)
    return out


def coded(m, r):
    """The values that the 8-bit state holds of m and sqrt v (64 bits that are fp32 values), blocks of 128."""
    out = []
    for x, top, least in ((m, 127.0, 0.0), (r, 255.0, 1.0)):
        x = x.view(-1, 128)
        most = x.abs().amax(1, keepdim=True)
        unit = f32(most * f32(torch.tensor(1 / top ** 2, dtype=torch.float64, device="cuda")))
        c = torch.round(f32(torch.sqrt(f32(x.abs() * f32(top ** 2 / most.clamp(min=EMPTY))))))
        c = torch.where(x != 0, c.clamp(min=least), 0.0)
        out.append(f32(torch.where(most >= EMPTY, c * c * x.sign() * unit, 0.0)).view(-1))
    return out[0], f32(out[1] * out[1])


class Plain:
    """The formulas on padded flat vectors."""

    def __init__(self, params, lr, betas, eps, decays, bits):
        self.p = [p.double().reshape(-1) for p in params]
        self.kind = params[0].dtype
        self.m = [torch.zeros_like(padded(p)) for p in self.p]
        self.v = [torch.zeros_like(m) for m in self.m]
        self.lr, self.b, self.eps, self.decays, self.bits, self.t = lr, betas, eps, decays, bits, 0

    def step(self, grads, scale=None):
        self.t += 1
        (b1, b2), bounds = self.b, []
        c = [f32(torch.tensor(x, dtype=torch.float64, device="cuda")) for x in (b1, 1 - b1, b2, 1 - b2)]
        for i, g in enumerate(grads):
            if g is None:
                bounds.append(None)
                continue
            g = padded(g.double())
            if scale is not None:
                g = f32(g * scale.double())
            m, v = self.m[i], self.v[i]
            if self.bits == 8:
                m = f32(f32(m * c[0]) + f32(g * c[1]))
                v = f32(f32(v * c[2]) + f32(f32(g * g) * c[3]))
                r = f32(v.sqrt())
                self.m[i], self.v[i] = coded(m, r)
            else:
                m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
                self.m[i], self.v[i] = m, v
                r = v.sqrt()
            size = m.abs() + 2 * (1 - b1) * g.abs()          # (at least beta1 |m| + (1 - beta1) |g|)
            n = self.p[i].numel()
            c1, root = 1 / (1 - b1 ** self.t), (r / math.sqrt(1 - b2 ** self.t) + self.eps)[:n]
            p = self.p[i] * (1 - self.lr * self.decays[i]) - self.lr * c1 * m[:n] / root
            bounds.append(4 * U * self.p[i].abs() + 16 * U * self.lr * c1 * size[:n] / root)
            self.p[i] = p
        return bounds

    def follow(self, params, moments=None):
        """Go on from what was computed, so that every step is compared by itself."""
        self.p = [p.double().reshape(-1) for p in params]
        if moments is not None:
            at = 0
            for i, m in enumerate(self.m):
                self.m[i], self.v[i] = (x[at:at + m.numel()].double() for x in moments)
                at += m.numel()


SETS = [[1], [128], [127, 129], [5, 2048, 2049, 1], [4096, 300, 7, 64 * 33], [10000] * 3 + [3] * 90, [1] * 2100 + [5000], [300_001]]


@pytest.mark.parametrize("sizes", SETS)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_steps(optim, sizes, bits, ptype, gtype):
    lr, betas, eps = 1e-2, (0.9, 0.99), 1e-8
    decays = [0.1 * (i % 3) for i in range(len(sizes))]
    params = [gaussian(i, n, scale=0.5, dtype=ptype) for i, n in enumerate(sizes)]
    copies = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") if i % 2 == 0 else None for i, n in enumerate(sizes)] if ptype == torch.float32 else None
    plain = Plain(params, lr, betas, eps, decays, bits)
    opt = optim.AdamW(params, lr=lr, betas=betas, eps=eps, weight_decay=decays, state_bits=bits, copies=copies)
    for t in range(4):
        grads = [gaussian(1000 * t + i, n, scale=10.0 ** (i % 5 - 3), dtype=gtype) for i, n in enumerate(sizes)]
        if t == 2 and len(sizes) > 1:
            grads[1] = None
        for g in grads[::3]:
            if g is not None:
                g[::3] = 0
        scale = torch.full((1,), 0.37, device="cuda") if t == 1 else None
        before = [p.clone() for p in params]
        old = [x.clone() for x in plain.m], [x.clone() for x in plain.v]
        bounds = plain.step(grads, scale)
        opt.step(grads, scale)
        for i, b in enumerate(bounds):
            if b is None:
                assert torch.equal(params[i], before[i])
                continue
            got, want = params[i].double(), plain.p[i]
            room = b + (torch.finfo(ptype).eps / 2 if ptype == torch.bfloat16 else U) * want.abs() + 1e-40
            assert ((got - want).abs() <= 1.01 * room).all(), (t, i, float(((got - want).abs() / room).max()))
            if copies and copies[i] is not None:
                assert torch.equal(copies[i], params[i].bfloat16())
        m, v = (x.double() for x in opt.moments())
        at = 0
        for i, n in enumerate(sizes):
            L = -(-n // 128) * 128
            gm, gv = m[at:at + L], v[at:at + L]
            at += L
            if bits == 8:
                assert torch.equal(gm, plain.m[i]) and torch.equal(gv, plain.v[i])
            elif bounds[i] is not None:
                g = padded(grads[i].double()) * (1 if scale is None else scale.double())
                assert ((gm - plain.m[i]).abs() <= 4 * U * (0.9 * old[0][i].abs() + 0.2 * g.abs())).all()
                assert ((gv - plain.v[i]).abs() <= 6 * U * plain.v[i] + 1e-44).all()
            assert (gm[n:] == 0).all() and (gv[n:] == 0).all()
        assert at == opt.values
        plain.follow(params, (m, v))
    assert opt.steps == 4


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_at_any_address_and_what_lies_beside_them(optim, bits):
    """Views that start at odd places of one buffer; nothing between them is touched."""
    for dtype in (torch.float32, torch.bfloat16):
        whole = torch.full((20000,), 7.0, dtype=dtype, device="cuda")
        spans = [(1, 130), (200, 333), (1001, 1002), (2048, 6148), (7003, 12000), (12001, 12009)]
        params = [whole[a:b] for a, b in spans]
        for i, p in enumerate(params):
            p.copy_(gaussian(i, p.numel()))
        apart = [p.clone() for p in params]
        a, b = (optim.AdamW(x, lr=0.01, state_bits=bits) for x in (params, apart))
        for t in range(2):
            grads = [gaussian(t * 10 + i, p.numel() + 3)[3:] for i, p in enumerate(params)]
            a.step(grads)
            b.step([g.clone() for g in grads])
        assert all(torch.equal(x, y) for x, y in zip(params, apart))
        for x, y in spans:
            whole[x:y] = 7
        assert (whole == 7).all()


def test_values_that_are_not_finite_stay_in_their_block(optim):
    p = gaussian(1, 1000)
    opt = optim.AdamW([p], state_bits=8)
    g = gaussian(2, 1000)
    g[200], g[500] = float("nan"), float("inf")
    opt.step([g])
    assert p[200].isnan() and p[500].isnan() and int(p.isnan().sum()) == 2
    m, v = opt.moments()
    inside = torch.zeros(1024, dtype=torch.bool, device="cuda")
    inside[128:256] = inside[384:512] = True
    assert torch.equal(m.isnan(), inside) and torch.equal(v.isnan(), inside)
    p32 = gaussian(1, 1000)
    opt = optim.AdamW([p32])
    opt.step([g])
    assert torch.equal(p32.isnan(), p.isnan())


def test_small_and_absent_gradients(optim):
    """Blocks below 2^-100 count as zero; rows that never had a gradient stay where they are (without decay)."""
    for bits in (8, 32):
        p = gaussian(1, 512)
        start = p.clone()
        opt = optim.AdamW([p], lr=0.1, weight_decay=0.0, state_bits=bits)
        g = torch.zeros(512, device="cuda")
        g[128:256] = 1e-35
        g[256:300] = 1.0
        for _ in range(3):
            opt.step([g])
        assert torch.equal(p[:128], start[:128]) and torch.equal(p[300:], start[300:])
        assert (p[128:256] - start[128:256]).abs().max() <= 1e-6 and ((start[256:300] - p[256:300]) - 0.3).abs().max() <= 1e-3
        m, v = opt.moments()
        assert (m[:128] == 0).all() and m.isfinite().all() and v.isfinite().all()
        if bits == 8:
            assert (m[128:256] == 0).all() and (v[128:256] == 0).all()


def test_moments_that_are_loaded(optim):
    """Zeros of either sign, and values over many orders of magnitude: coded as the definition says."""
    n = 128 * 40
    m, v = gaussian(1, n) * torch.exp(3 * gaussian(2, n)), (gaussian(3, n) * torch.exp(3 * gaussian(4, n))) ** 2
    m[::3], v[::5], v[1::5] = -0.0, 0.0, -0.0
    m[128:256], v[256:384] = 0.0, -0.0
    m[384:512] *= 1e-36
    v[384:512] *= 1e-30
    v[512:640] *= 1e-34                                      # roots of numbers near the least normal one
    v[640:650] = 1e-44
    opt = optim.AdamW([torch.zeros(n, device="cuda")], state_bits=8)
    opt.load_moments(7, m, v)
    want = coded(m.double(), f32(v.double().abs().sqrt()))
    got = opt.moments()
    assert torch.equal(got[0].double(), want[0]) and torch.equal(got[1].double(), want[1]) and opt.steps == 7


def test_states_go_out_and_back(optim):
    sizes = [1000, 77, 5000]
    for bits in (8, 32):
        params = [gaussian(i, n) for i, n in enumerate(sizes)]
        opt = optim.AdamW(params, lr=0.01, state_bits=bits)
        for t in range(3):
            opt.step([gaussian(10 * t + i, n) for i, n in enumerate(sizes)])
        kept, d = [p.clone() for p in params], opt.state_dict()
        m, v = (x.clone() for x in opt.moments())
        other = [p.clone() for p in kept]
        again = optim.AdamW(other, lr=0.5, state_bits=bits)
        again.load_state_dict(d)
        third = [p.clone() for p in kept]
        from_moments = optim.AdamW(third, lr=0.01, state_bits=bits)
        from_moments.load_moments(3, m, v)
        if bits == 8:                                        # the codes' own values are coded as themselves
            assert all(torch.equal(a, b) for a, b in zip(from_moments._state[:2], opt._state[:2]))
        g = [gaussian(99 + i, n) for i, n in enumerate(sizes)]
        for o in (opt, again, from_moments):
            o.step(g)
        assert all(torch.equal(a, b) for a, b in zip(params, other)) and again.steps == 4 and again.lr == 0.01
        assert all((a - b).abs().max() <= 1e-6 for a, b in zip(params, third))
        with pytest.raises(ValueError):
            optim.AdamW(other, state_bits=40 - bits).load_state_dict(d)


def test_what_autograd_kept_of_a_parameter_is_not_used_after_a_step(optim):
    w = torch.nn.Parameter(gaussian(1, 30))
    opt = optim.AdamW([w])
    y = (w * w).sum()
    opt.step([gaussian(2, 30)])
    with pytest.raises(RuntimeError):
        y.backward()
    (w * w).sum().backward()
    opt.step()


def test_an_optimizer_is_not_copied(optim):
    import copy
    import pickle
    opt = optim.AdamW([gaussian(1, 30)])
    for f in (copy.copy, copy.deepcopy, pickle.dumps):
        with pytest.raises(TypeError):
            f(opt)


def test_captured_steps_count_their_replays_and_follow_the_rate(optim):
    sizes = [3000, 10, 777]
    for bits in (8, 32):
        a, b = ([gaussian(i, n) for i, n in enumerate(sizes)] for _ in range(2))
        grads = [torch.zeros(n, device="cuda") for n in sizes]
        x, y = optim.AdamW(a, lr=0.01, state_bits=bits), optim.AdamW(b, lr=0.01, state_bits=bits)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            x.step(grads)
        for t in range(4):
            for i, g in enumerate(grads):
                g.copy_(gaussian(50 * t + i, g.numel()))
            if t == 2:
                x.lr = y.lr = 0.003
            graph.replay()
            y.step(grads)
            assert all(torch.equal(p, q) for p, q in zip(a, b))
        assert x.steps == y.steps == 4


def test_gradients_of_torch_and_agreement_with_its_own_optimizer(optim):
    """The same model by torch.optim.AdamW in 64 bits."""
    w = [torch.nn.Parameter(gaussian(1, 40, 30)), torch.nn.Parameter(gaussian(2, 40))]
    d = [torch.nn.Parameter(p.detach().double().clone()) for p in w]
    opt, ref = optim.AdamW(w, lr=0.01, weight_decay=0.05), torch.optim.AdamW(d, lr=0.01, weight_decay=0.05)
    for t in range(5):
        x = gaussian(10 + t, 64, 30)
        for p in w + d:
            p.grad = None
        (x @ w[0].t() + w[1]).tanh().square().sum().backward()
        for p, q in zip(w, d):
            q.grad = p.grad.double()
        opt.step()
        ref.step()
    for p, q in zip(w, d):
        assert float((p.detach().double() - q.detach()).abs().max()) <= 5 * 24 * U * 3      # five steps; |p| < 3 or so, updates of 0.01


@pytest.mark.parametrize("bits", [8, 32])
def test_a_model_trains_with_8_bits_as_with_32(optim, bits):
    """Minimises |x - c|^2 from far away under noise: both come as near as the rate lets them."""
    n = 5000
    c = gaussian(3, n) * torch.exp(gaussian(4, n))
    x = torch.zeros(n, device="cuda")
    opt = optim.AdamW([x], lr=0.05, betas=(0.9, 0.99), weight_decay=0.0, state_bits=bits)
    for t in range(600):
        if t == 400:
            opt.lr = 0.005
        opt.step([(x - c) + gaussian(t, n, scale=0.1)])
    near = c.abs() < 10
    assert float((x - c)[near].abs().mean()) <= 0.05


def test_more_tensors_than_a_launch_takes_is_one_step(optim):
    sizes = [3] * 2500
    p = [gaussian(i, n) for i, n in enumerate(sizes)]
    one = torch.cat(p)
    a, b = optim.AdamW(p, lr=0.1), optim.AdamW([one], lr=0.1)
    for t in range(3):
        g = gaussian(t, 7500)
        a.step(list(g.split(3)))
        b.step([g])
    assert torch.equal(torch.cat(p), one) and a.steps == 3 and a.launch_count == 9


def test_more_than_2_to_the_31_values(optim):
    n = 2 ** 31 + 5000
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    opt = optim.AdamW([p], lr=0.125, weight_decay=0.0, state_bits=8)
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    g[-3000:] = -1
    opt.step([g])
    assert (p[-3000:] == 0.125).all() and (p[:-3000] == -0.125).all()


# ------------------------------------------------------------------------------------------------------- the engine's workers
@pytest.mark.parametrize("K,P", [(1, 7), (3, 1000), (4, 5003), (2, 70000)])
@pytest.mark.parametrize("bits", [8, 32])
def test_local_steps_of_the_workers(optim, K, P, bits):
    """A round with AdamW local steps: the same as K optimizers by themselves, the mean and the merge the engine's own; right after the round's begin
    the step writes the other buffer."""
    from paper_1906_12043_b200 import engine as E
    eng = E.Engine(K, P, 0.1, 0.9, 0.0)
    eng.set_option(E.OPT_BF16_SHADOW, 1)
    x0 = gaussian(1, K, P)
    eng.set_params_all(x0)
    tensors = [(P // 2, 0.1), (P // 3, 0.0)] if P > 10 else None
    opt = optim.EngineAdamW(eng, tensors, lr=0.01, state_bits=bits)
    whole = [n for n, _ in tensors] + [P - sum(n for n, _ in tensors)] if tensors else [P]
    models = [x0[i].clone() for i in range(K)]
    alone = [optim.AdamW(list(m.split(whole)), lr=0.01, weight_decay=[d for _, d in tensors] + [0.0] if tensors else 0.0, state_bits=bits) for m in models]
    side = torch.cuda.Stream(priority=-1)
    for r in range(2):
        stored = eng.get_params()
        eng.comm_begin(side)
        for s in range(3):
            g = gaussian(10 * r + s, K, P)
            opt.local_step(g)
            for i in range(K):
                alone[i].step(list(g[i].split(whole)))
            eng.sync()
            x = eng.get_params()
            assert torch.equal(x, torch.stack(models)) and torch.equal(eng.bf16_shadow(), x.bfloat16())
        eng.comm_end()
        eng.sync()
        x, mean = eng.get_params(), eng.get_mean()
        assert torch.equal(x, mean + (torch.stack(models) - stored)) and (mean.double() - stored.double().mean(0)).abs().max() <= 1e-6
        for i in range(K):
            models[i].copy_(x[i])
    assert opt.steps == 6 and eng.step_count == 6


def test_an_engine_on_a_stream_of_its_own(optim):
    """Rates, moments and steps are ordered with the engine's calls."""
    from paper_1906_12043_b200 import engine as E
    K, P = 2, 300_000
    s = torch.cuda.Stream()
    for bits in (8, 32):
        x0, g = gaussian(1, K, P), gaussian(2, K, P)
        torch.cuda.synchronize()
        got = []
        for stream in (s, None):
            eng = E.Engine(K, P, 0.1, 0.9, 0.0, stream=stream)
            eng.set_params_all(x0)
            opt = optim.EngineAdamW(eng, lr=0.01, state_bits=bits)
            for t in range(6):
                opt.local_step(g)
                opt.lr = 0.01 * (t + 1)
            d = opt.state_dict()
            opt.load_state_dict(d)
            m, v = opt.moments()
            eng.sync()
            torch.cuda.synchronize()
            got.append((eng.get_params(), m.clone(), v.clone()))
            eng.sync()
            assert opt.steps == 6
        assert all(torch.equal(a, b) for a, b in zip(*got))


def test_refusals(optim):
    from paper_1906_12043_b200 import engine as E
    p = [gaussian(1, 10), gaussian(2, 20)]
    g = [gaussian(3, 10), gaussian(4, 20)]
    for bad in (dict(params=[]), dict(params=[1]), dict(params=[p[0], p[0]]), dict(state_bits=16), dict(weight_decay=[0.1]), dict(copies=[None]),
                dict(copies=[p[0].clone(), None], params=[x.bfloat16() for x in p]), dict(params=[p[0], torch.empty(0, device="cuda")])):
        with pytest.raises(ValueError):
            optim.AdamW(**{"params": p, **bad})
    for bad in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(lr=float("nan")), dict(weight_decay=float("inf"))):
        with pytest.raises(E.CocodError):
            optim.AdamW(p, **bad)
    opt = optim.AdamW(p)
    before = [x.clone() for x in p]
    wide = torch.zeros(20, 2, device="cuda")[:, 0]
    for bad in (g[:1], [g[0], g[0]], [g[0].double(), g[1].double()], [g[0], g[1].bfloat16()], [g[0].cpu(), g[1]], [g[0], wide], [p[0], g[1]], [g[0], 1]):
        with pytest.raises(ValueError):
            opt.step(bad)
    for bad in (torch.ones(2, device="cuda"), torch.ones(1), torch.ones(1, device="cuda", dtype=torch.float64), 0.5):
        with pytest.raises(ValueError):
            opt.step(g, bad)
    m, v = opt.moments()
    for bad in ((-1, m, v), (0, m[1:], v), (0, m.double(), v), (0, m, v.cpu())):
        with pytest.raises(ValueError):
            opt.load_moments(*bad)
    with pytest.raises(E.CocodError):
        opt.lr = float("nan")
    with pytest.raises(ValueError):
        optim.AdamW(p, copies=[torch.zeros(10, device="cuda"), None]).step(g)
    assert all(torch.equal(a, b) for a, b in zip(p, before)) and opt.steps == 0
    eng = E.Engine(2, 100, 0.1, 0.9, 0.0)
    for bad in ([(101, 0.0)], [(0, 0.0)]):
        with pytest.raises(ValueError):
            optim.EngineAdamW(eng, bad)
    with pytest.raises(ValueError):
        optim.EngineAdamW(eng).local_step(torch.zeros(2, 99, device="cuda"))
    other = E.Engine(2, 128, 0.1, 0.9, 0.0)
    mine = optim.EngineAdamW(eng)
    mine.engine = other
    with pytest.raises(E.CocodError):
        mine.local_step(torch.zeros(2, 128, device="cuda"))
    mine.destroy()
    with pytest.raises(ValueError):
        mine.local_step(torch.zeros(2, 128, device="cuda"))
    opt.destroy()
    with pytest.raises(ValueError):
        opt.step(g)


def queue_work(ms=30):
    """Ordinary work that keeps the current stream busy for a while (a product of 8192^3 takes more than 0.7 ms)."""
    a = torch.ones(8192, 8192, dtype=torch.bfloat16, device="cuda")
    for _ in range(int(ms / 0.7)):
        torch.mm(a, a)


@pytest.mark.parametrize("bits", [8, 32])
def test_an_engine_on_a_stream_of_its_own_and_a_busy_current_stream(optim, bits):
    """The zeros of a new state, copies of the state and moments that are handed out or in come from the current stream: the engine's steps and they wait for each other."""
    from paper_1906_12043_b200 import engine as E
    K, P = 2, 3_000_001
    x0, g = gaussian(1, K, P), gaussian(2, K, P)
    torch.cuda.synchronize()
    got = []
    for stream in (None, torch.cuda.Stream()):
        busy = queue_work if stream is not None else lambda: None
        eng = E.Engine(K, P, 0.1, 0.9, 0.0, stream=stream)
        eng.set_params_all(x0)
        torch.cuda.synchronize()
        busy()
        opt = optim.EngineAdamW(eng, lr=0.01, state_bits=bits)
        opt.local_step(g)
        opt.local_step(g)
        busy()
        d = opt.state_dict()
        opt.local_step(g)
        seen = [t.clone() for t in d["state"]]
        busy()
        opt.load_state_dict(d)
        for t in d["state"]:                                 # (what was read may be changed)
            t.zero_()
        opt.local_step(g)
        busy()
        before = [torch.full((opt.values,), 7.0, device="cuda") for _ in range(2)]
        del before                                           # (the next results may lie where this is still being written)
        moments = [t.clone() for t in opt.moments()]
        opt.local_step(g)
        busy()
        m, v = (t * 2 for t in moments)
        opt.load_moments(5, m, v)
        m.zero_(), v.zero_()
        opt.local_step(g)
        eng.sync()
        torch.cuda.synchronize()
        got.append([eng.get_params(), *seen, *moments, *(t.clone() for t in opt.moments())])
        torch.cuda.synchronize()
        assert opt.steps == 6
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("n", [3, 70])
def test_tensors_of_other_sizes_than_the_state_are_refused(optim, bits, n):
    """The kernels go by the sizes given at creation: a parameter that was taken out, shortened or lengthened since is refused before anything is read or written."""
    for change in ("fewer", "more", "shorter", "longer", "a shorter copy", "a longer gradient"):
        params = [torch.nn.Parameter(gaussian(i, 300)) for i in range(n)]
        opt = optim.AdamW(params, state_bits=bits, copies=[p.detach().bfloat16() for p in params])
        opt.step([gaussian(i, 300) for i in range(n)])
        grads = [gaussian(i, 300) for i in range(n)]
        with pytest.raises((AttributeError, TypeError)):
            opt.params.pop()
        if change == "fewer":
            opt.params, opt.copies = opt.params[:-1], opt.copies[:-1]
            grads.pop()
        elif change == "more":
            opt.params, opt.copies = opt.params + (gaussian(1, 300),), opt.copies + (None,)
            grads.append(gaussian(2, 300))
        elif change == "a shorter copy":
            opt.copies = opt.copies[:-1] + (opt.copies[-1][:299],)
        else:
            size = 299 if change == "shorter" else 301
            if change != "a longer gradient":
                params[-1].data = gaussian(1, size)
            grads[-1] = gaussian(2, size)
        kept = [p.detach().clone() for p in params] + [t.clone() for t in opt.moments()]
        with pytest.raises(ValueError):
            opt.step(grads)
        with pytest.raises(ValueError):
            opt.step(tuple(grads))
        assert all(torch.equal(a, b) for a, b in zip(kept, [p.detach() for p in params] + list(opt.moments()))) and opt.steps == 1


@pytest.mark.parametrize("bits", [8, 32])
def test_a_state_that_is_refused_changes_nothing(optim, bits):
    p = [gaussian(1, 300)]
    opt, other = optim.AdamW(p, state_bits=bits), optim.AdamW([gaussian(1, 300)], state_bits=bits)
    for o in (opt, other):
        o.step([gaussian(2, 300)])
    other.step([gaussian(3, 300)])
    kept = [t.clone() for t in opt.moments()]
    d = other.state_dict()
    for bad in (dict(d, steps=-1), dict(d, lr=float("nan")), dict(d, lr=float("inf")), dict(d, state=d["state"][:1]), dict(d, state_bits=40 - bits)):
        with pytest.raises(ValueError):
            opt.load_state_dict(bad)
        assert all(torch.equal(a, b) for a, b in zip(kept, opt.moments())) and opt.steps == 1
    opt.load_state_dict(d)
    assert all(torch.equal(a, b) for a, b in zip(other.moments(), opt.moments())) and opt.steps == 2


LARGE = [[1_000_003, 150 * 4096 + 5, 7, 300_000], [40_000_000, 333, 5_000_001]]


@pytest.mark.parametrize("sizes", LARGE)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("ptype,gtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_steps_of_large_models(optim, sizes, bits, ptype, gtype):
    """Chunks of 4096 values and more, whose 8-bit form loads a step ahead: three steps against the formulas, by the bounds above."""
    lr, betas, eps, decays = 1e-2, (0.9, 0.99), 1e-8, [0.1 * (i % 3) for i in range(len(sizes))]
    params = [gaussian(i, n, scale=0.5, dtype=ptype) for i, n in enumerate(sizes)]
    plain = Plain(params, lr, betas, eps, decays, bits)
    opt = optim.AdamW(params, lr=lr, betas=betas, eps=eps, weight_decay=decays, state_bits=bits)
    for t in range(3):
        grads = [gaussian(1000 * t + i, n, scale=10.0 ** (i % 5 - 3), dtype=gtype) for i, n in enumerate(sizes)]
        grads[0][::3] = 0
        old = [x.clone() for x in plain.m]
        bounds = plain.step(grads)
        opt.step(grads)
        m, v = opt.moments()
        at = 0
        for i, n in enumerate(sizes):
            got, want = params[i].double(), plain.p[i]
            room = bounds[i] + (torch.finfo(ptype).eps / 2 if ptype == torch.bfloat16 else U) * want.abs() + 1e-40
            assert ((got - want).abs() <= 1.01 * room).all(), (t, i)
            L = -(-n // 128) * 128
            gm, gv = m[at:at + L].double(), v[at:at + L].double()
            at += L
            if bits == 8:
                assert torch.equal(gm, plain.m[i]) and torch.equal(gv, plain.v[i])
            else:
                assert ((gm - plain.m[i]).abs() <= 4 * U * (0.9 * old[i].abs() + 0.2 * padded(grads[i].double()).abs())).all()
                assert ((gv - plain.v[i]).abs() <= 6 * U * plain.v[i] + 1e-44).all()
            assert (gm[n:] == 0).all() and (gv[n:] == 0).all()
        plain.follow(params, (m, v))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("first", [128, 10])
def test_local_steps_of_large_models(optim, bits, first):
    """The workers' tensors one behind the other, all of them aligned or, behind ten values, none: the same bits as lists of tensors."""
    from paper_1906_12043_b200 import engine as E
    K, sizes = 3, [first, 1_500_000, 2047, 400_000]
    P = sum(sizes)
    x0 = gaussian(1, K, P)
    eng = E.Engine(K, P, 0.1, 0.9, 0.0)
    eng.set_params_all(x0)
    opt = optim.EngineAdamW(eng, [(n, 0.1 * (i % 2)) for i, n in enumerate(sizes)], lr=0.01, state_bits=bits)
    tensors = [t.clone() for i in range(K) for t in x0[i].split(sizes)]
    alone = optim.AdamW(tensors, lr=0.01, weight_decay=[0.1 * (i % 2) for i in range(len(sizes))] * K, state_bits=bits)
    for t in range(3):
        g = gaussian(10 + t, K, P)
        opt.local_step(g)
        alone.step([p.clone() for i in range(K) for p in g[i].split(sizes)])
    eng.sync()
    x = eng.get_params()
    assert torch.equal(x.view(-1), torch.cat(tensors)) and all(torch.equal(a, b) for a, b in zip(opt.moments(), alone.moments()))
