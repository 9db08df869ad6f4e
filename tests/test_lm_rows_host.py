"""Experts, log probabilities and AdamW without a GPU: refusals at the C boundary and of the binding, and sizes."""
import ctypes

import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    from paper_1906_12043_b200 import build, engine
    build.build()
    return engine.load()


def test_calls_without_a_handle_are_refused(lib):
    from paper_1906_12043_b200.engine import ERR_INVALID, OK
    assert lib.cocod_expert_sort(None, 1, 1, 1, 16, 1, 16, 16, 16, 16, None, 0, None) == ERR_INVALID
    assert lib.cocod_expert_rows(None, 1, 1, 8, 16, 8, 16, 16, 8, 0, None) == ERR_INVALID
    assert lib.cocod_expert_join(None, 1, 1, 8, 16, 8, 0, 16, 16, 16, 8, 0, None) == ERR_INVALID
    assert lib.cocod_expert_join_grad(None, 1, 1, 8, 16, 8, 16, 8, 16, 16, 16, 8, 16, 0, None) == ERR_INVALID
    assert lib.cocod_token_logprobs(None, 1, 8, 16, 8, 1, None, 1.0, 0, 16, 16, 16, None, None, None) == ERR_INVALID
    assert lib.cocod_token_logprobs_grad(None, 1, 8, 16, 8, 1, None, 1.0, 0, None, 16, 16, None, 16, None, 16, 8, None) == ERR_INVALID
    assert lib.cocod_adamw_destroy(None) == OK
    assert lib.cocod_adamw_step(None, None, 1, None, 1, None, None, None) == ERR_INVALID
    assert lib.cocod_adamw_flat_step(None, 16, 16, 1, 16, 1, None, None, None) == ERR_INVALID
    assert lib.cocod_adamw_local_step(None, None, None, None) == ERR_INVALID
    assert lib.cocod_adamw_set_lr(None, 1.0, None) == ERR_INVALID
    assert lib.cocod_adamw_set_step(None, 1, None) == ERR_INVALID
    assert lib.cocod_adamw_get_step(None, None, None) == ERR_INVALID
    assert lib.cocod_adamw_moments(None, 16, 16, None) == ERR_INVALID
    assert lib.cocod_adamw_load(None, 16, 16, None) == ERR_INVALID
    assert lib.cocod_adamw_launch_count(None) == -1


@pytest.mark.parametrize("T,k,E", [(-1, 1, 1), (1, 0, 1), (1, 33, 40), (1, 1, 0), (1, 1, 1025), (2 ** 31, 1, 4), (2 ** 27, 16, 4)])
def test_sizes_of_experts_out_of_range(lib, T, k, E):
    assert lib.cocod_expert_workspace(T, k, E) < 0


def test_workspaces_of_the_sort(lib):
    """Few slots need none, and no number of slots needs more than counts for a thread block on every SM and a cluster of them."""
    assert lib.cocod_expert_workspace(0, 1, 1) == lib.cocod_expert_workspace(1, 1, 1024) == lib.cocod_expert_workspace(64, 32, 7) == 0
    for T in (5000, 10 ** 6, 2 ** 31 - 2000):
        assert 0 < lib.cocod_expert_workspace(T, 1, 100) <= 148 * 9 // 8 * 101 * 4


def sizes(*n):
    return len(n), (ctypes.c_int64 * max(1, len(n)))(*n)


def test_values_of_the_moments(lib):
    assert lib.cocod_adamw_values(*sizes(1)) == 128 and lib.cocod_adamw_values(*sizes(128, 129, 1)) == 512
    for bad in (sizes(), sizes(0), sizes(5, -1), sizes(2 ** 40), sizes(*[2 ** 39] * 3), (1, None), (-1, sizes(1)[1])):
        assert lib.cocod_adamw_values(*bad) < 0


def test_adamw_is_looked_over_before_anything_is_made(lib):
    from paper_1906_12043_b200.engine import ERR_INVALID
    out, nan, inf = ctypes.c_void_p(), float("nan"), float("inf")
    good = dict(out=ctypes.byref(out), n=2, sizes=sizes(3, 4)[1], decay=None, starts=None, bits=8, m=256, v=256, mu=256, vu=256, lr=0.1, b1=0.9, b2=0.99, eps=1e-8)
    decays = (ctypes.c_float * 2)
    starts = (ctypes.c_int64 * 2)
    for bad in (dict(out=None), dict(n=0), dict(sizes=None), dict(sizes=sizes(3, 0)[1]), dict(bits=16), dict(bits=0), dict(m=None), dict(v=None), dict(m=8), dict(mu=None),
                dict(vu=None), dict(vu=2), dict(lr=nan), dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1.0), dict(eps=nan), dict(eps=inf),
                dict(decay=decays(0.1, nan)), dict(starts=starts(0, -1))):
        assert lib.cocod_adamw_create(*{**good, **bad}.values()) == ERR_INVALID, bad
    assert not out.value


def test_operators_refuse_to_run_without_a_gpu(lib):
    from paper_1906_12043_b200 import optim
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        optim.AdamW([torch.zeros(3)])


def test_the_binding_refuses_without_a_gpu(lib):
    from paper_1906_12043_b200 import _lm_binding as b
    for f, n in (("expert_sort", 4), ("expert_rows", 5), ("expert_join", 7), ("expert_join_grad", 7), ("token_logprobs", 6), ("token_logprobs_grad", 12), ("adamw_step", 6),
                 ("adamw_moments", 5)):
        with pytest.raises(ValueError, match="number of arguments"):
            getattr(b, f)(*[0] * (n - 1))
        with pytest.raises(ValueError, match="destroyed"):
            getattr(b, f)(*[0] * n)


def test_the_measured_cases_are_of_their_ranges():
    """perf/more_operators.py: names, work and draws, without a GPU."""
    import importlib.util
    import os
    import random
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    spec = importlib.util.spec_from_file_location("more_operators", os.path.join(root, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    listed = m.listed()
    assert len({c["name"] for c in listed}) == len(listed) and not m.own
    rng = random.Random(1)
    most = max(m.work(c)["bytes"] for c in listed)
    for c in listed + [m.draw(rng) for _ in range(200)]:
        assert 0 < m.work(c)["bytes"] <= most


class FakeStream:
    def __init__(self, at, log):
        self.cuda_stream, self.log = at, log

    def wait_stream(self, other):
        self.log.append((self.cuda_stream, "waits for", other.cuda_stream))


def test_an_engines_optimizer_orders_its_stream_with_the_current_one(lib, monkeypatch):
    """Every tensor that goes in or out, and the zeros of the new state: the engine's stream (7) waits for the current one (5) before, the current one for it after."""
    import contextlib
    from types import SimpleNamespace

    from paper_1906_12043_b200 import _lm_binding, engine, optim
    log, here = [], None

    class Library:
        def __getattr__(self, name):
            def call(*a):
                log.append(name)
                if name == "cocod_adamw_create":
                    a[0]._obj.value = 1
                return 256 if name == "cocod_adamw_values" else 0
            return call

    @contextlib.contextmanager
    def stream(s):
        log.append(("on", s.cuda_stream))
        yield
        log.append("off")

    here = FakeStream(5, log)
    zeros = torch.zeros
    for name, f in (("is_available", lambda: True), ("current_device", lambda: 0), ("current_stream", lambda: here), ("stream", stream), ("ExternalStream", lambda at: FakeStream(at, log))):
        monkeypatch.setattr(torch.cuda, name, f)
    monkeypatch.setattr(torch, "zeros", lambda *a, device, **k: log.append("zeros") or zeros(*a, **k))
    monkeypatch.setattr(engine, "load", Library)
    monkeypatch.setattr(_lm_binding, "adamw_moments", lambda *a: log.append(("moments", a[-1])) or (zeros(256),) * 2)
    monkeypatch.setattr(optim._Moments, "_flat", lambda self, t, name: t.data_ptr())
    first, last = (7, "waits for", 5), (5, "waits for", 7)
    e = SimpleNamespace(K=2, P=100, _compute=7, _h=1)
    for bits in (8, 32):
        log.clear()
        opt = optim.EngineAdamW(e, state_bits=bits)
        assert log.index("zeros") < log.index(first)
        log.clear()
        d = opt.state_dict()
        assert log == ["cocod_adamw_get_step", first, ("on", 7), "off", last]
        log.clear()
        opt.load_state_dict(d)
        assert log[:4] == [first, ("on", 7), "off", last]
        log.clear()
        opt.load_moments(1, *(zeros(256),) * 2)
        assert log[:3] == [first, "cocod_adamw_load", last]
        log.clear()
        opt.moments()
        assert log == [first, ("moments", 7), last]
        here.cuda_stream = 7                                 # (the same stream: nothing to wait for)
        log.clear()
        opt.moments()
        assert log == [("moments", 7)]
        here.cuda_stream = 5


def test_no_sizes_without_a_handle(lib):
    n = ctypes.c_int(5)
    assert not lib.cocod_adamw_sizes(None, ctypes.byref(n)) and n.value == 5


def test_an_engines_optimizer_refuses_tensors_of_another_device(monkeypatch):
    """... before their addresses get to a kernel."""
    from types import SimpleNamespace

    from paper_1906_12043_b200 import optim
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    opt = optim.EngineAdamW.__new__(optim.EngineAdamW)
    called = []
    opt._h, opt._device = 1, 0
    opt._lib = SimpleNamespace(cocod_adamw_local_step=lambda *a: called.append(a) or 0, cocod_adamw_destroy=lambda h: 0)
    opt.engine = SimpleNamespace(K=1, P=4, _h=1, _compute=7, _check_tensor=lambda *a: 0)

    def on(device, n):
        return SimpleNamespace(get_device=lambda: device, is_cuda=True, dtype=torch.float32, numel=lambda: n, data_ptr=lambda: 256)

    opt.local_step(on(0, 4), on(0, 1))
    assert len(called) == 1
    for bad in ((on(1, 4), None), (on(0, 4), on(1, 1))):
        with pytest.raises(ValueError, match="cuda:1"):
            opt.local_step(*bad)
    assert len(called) == 1
