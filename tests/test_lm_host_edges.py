"""The language-model operators' host side, without a GPU: copies of checkpoints, and how workspaces follow their limit."""
import copy
import pickle

import pytest

torch = pytest.importorskip("torch")


def checkpoint(M, k):
    from paper_1906_12043_b200 import lm
    ld, blocks = -(-k // 16) * 16, -(-k // 128)
    return lm.PackedActivations._of(torch.randint(0, 256, (M * ld + blocks * M,), dtype=torch.uint8), M, k)


@pytest.mark.parametrize("M,k", [(1, 1), (5, 200), (3, 128), (0, 40)])
def test_a_copy_of_a_checkpoint_reads_its_own_memory(M, k):
    first = checkpoint(M, k)
    again = type(first).from_parts(first.q.clone() if M == 1 else first.q, first.scales)
    for p in (first, again):
        for q in (copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
            assert torch.equal(q.q, p.q) and torch.equal(q.scales, p.scales) and q.shape == p.shape and q._ld == p._ld
            assert q._at == q.q.data_ptr() and q._scales_at == q.scales.data_ptr()
            assert M == 0 or (q._at != p._at and q._scales_at != p._scales_at)


@pytest.mark.parametrize("G,M,V,D", [(1, 1, 1, 8), (1, 300, 1000, 64), (1, 8192, 65536, 2048), (16, 2048, 16384, 1024), (4, 70001, 50001, 768)])
@pytest.mark.parametrize("grad", [0, 1])
@pytest.mark.parametrize("dw_type", [0, 1])
def test_workspaces_rise_with_their_limit_and_stay_within_it(G, M, V, D, grad, dw_type):
    """... unless not even the fewest rows fit, and then they are those of the fewest rows."""
    from paper_1906_12043_b200 import build, engine
    build.build()
    f = engine.load().cocod_vocab_workspace
    whole, least = f(G, M, V, D, grad, dw_type, 1 << 60), f(G, M, V, D, grad, dw_type, 0)
    last = 0
    for limit in sorted({0, least - 1, least, least + 1, whole - 1, whole, whole + 1} | {whole * i // 23 for i in range(1, 24)}):
        got = f(G, M, V, D, grad, dw_type, limit)
        assert got >= last and (got <= limit or got == least)
        assert limit < whole or got == whole
        last = got


def test_the_binding_loads_and_refuses_without_a_gpu():
    from paper_1906_12043_b200 import build
    build.build()
    from paper_1906_12043_b200 import _lm_binding
    with pytest.raises(ValueError, match="destroyed"):
        _lm_binding.act_pack_new(0, 0, torch.zeros(1, 1))
    with pytest.raises(ValueError, match="number of arguments"):
        _lm_binding.act_pack_new(0)
