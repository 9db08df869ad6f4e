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
