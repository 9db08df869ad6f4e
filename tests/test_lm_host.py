"""The language-model operators' host side, without a GPU: refusals, and the sizes of workspaces."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def lib():
    from paper_1906_12043_b200 import build, engine
    build.build()
    return engine.load()


def test_calls_without_a_handle_are_refused(lib):
    from paper_1906_12043_b200.engine import ERR_INVALID, OK
    assert lib.cocod_lm_create(None) == ERR_INVALID
    assert lib.cocod_lm_destroy(None) == OK
    assert lib.cocod_lm_check(None, None) == ERR_INVALID
    assert lib.cocod_lm_launch_count(None) == -1
    for f in (lib.cocod_grouped_forward, lib.cocod_grouped_input_grad):
        assert f(None, 1, 16, 8, 8, 8, 16, 8, 16, 8, 64, 16, 8, 0, None) == ERR_INVALID
    assert lib.cocod_grouped_weight_grad(None, 1, 16, 8, 8, 8, 16, 8, 16, 8, 16, 8, 64, 0, None) == ERR_INVALID
    assert lib.cocod_grouped_weight_grad_packed(None, 1, 16, 8, 8, 8, 16, 8, 16, 16, 16, 16, 8, 64, 0, None, 0, None) == ERR_INVALID
    assert lib.cocod_act_pack(None, 1, 8, 16, 8, 16, 16, 16, None) == ERR_INVALID
    assert lib.cocod_act_unpack(None, 1, 8, 16, 16, 16, 16, 8, None) == ERR_INVALID
    assert lib.cocod_act_relu_grad(None, 1, 8, 16, 8, 16, 16, 16, 8, None) == ERR_INVALID
    assert lib.cocod_vocab_loss(None, 1, 16, 8, 8, 8, 16, 8, 16, 8, 64, 16, None, 16, 16, 256, 1 << 20, None) == ERR_INVALID
    assert lib.cocod_vocab_loss_grad(None, 1, 16, 8, 8, 8, 16, 8, 16, 8, 64, 16, None, 16, 16, 16, 8, 16, 8, 64, 0, 256, 1 << 20, None) == ERR_INVALID
    for ms in (0, -1, 2001):
        assert lib.cocod_grouped_wait_selftest(ms, 0, None) == ERR_INVALID


def test_sizes_out_of_range_are_refused(lib):
    assert lib.cocod_grouped_packed_workspace(0, 8, 8, 8) < 0
    for args in ((0, 8, 8, 8, 1, 0, 0), (1, -1, 8, 8, 1, 0, 0), (1, 8, 0, 8, 1, 0, 0), (1, 8, 8, 12, 1, 0, 0), (1, 8, 8, 8, 1, 2, 0), (1, 8, 8, 8, 1, 0, -1)):
        assert lib.cocod_vocab_workspace(*args) < 0


@pytest.mark.parametrize("G,M,V,D", [(1, 1, 1, 8), (1, 8192, 65536, 2048), (16, 2048, 16384, 1024), (4, 70001, 50001, 768)])
@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("dw_type", [0, 1])
def test_vocabulary_workspace_keeps_to_its_limit(lib, G, M, V, D, grad, dw_type):
    whole = lib.cocod_vocab_workspace(G, M, V, D, grad, dw_type, 1 << 60)
    least = lib.cocod_vocab_workspace(G, M, V, D, grad, dw_type, 0)
    assert 0 < least <= whole
    last = 0
    for limit in (0, whole // 8, whole // 3, whole // 2, whole, 2 * whole):
        got = lib.cocod_vocab_workspace(G, M, V, D, grad, dw_type, limit)
        assert got <= max(limit, least) or got <= whole
        assert got >= min(last, least)
        last = got
    if grad:
        # the exponentials of 256 rows at the least, of all rows at the most (several passes also need the fp32 sums of a bf16 gradient)
        assert least >= 2 * min(M, 256) * V and whole >= 2 * M * V
    else:
        assert whole <= 64 * M + M * V // 4 + 65536       # two numbers for each row and 64 entries


def test_operators_refuse_to_run_without_a_gpu(lib):
    from paper_1906_12043_b200 import lm
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(RuntimeError):
        lm.LMOps()


def test_a_checkpoint_made_elsewhere_is_looked_at():
    from paper_1906_12043_b200 import lm
    q = torch.zeros(5, 208, dtype=torch.int8)[:, :200]
    s = torch.zeros(2, 5, dtype=torch.uint8)
    p = lm.PackedActivations.from_parts(q, s)
    assert p.shape == (5, 200) and p.q is q and p.scales is s
    for bad_q, bad_s in ((q.to(torch.uint8), s), (q, s.to(torch.int8)), (q, s[:1]), (q.contiguous(), s), (q, s.t().contiguous().t()), (q[:, 1:], s)):
        with pytest.raises(ValueError):
            lm.PackedActivations.from_parts(bad_q, bad_s)
