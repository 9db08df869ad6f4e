"""The example of workers that train a next-token model: its gradients against 64 bits, and that it learns."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_1906_12043_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location("lm_workers", os.path.join(ROOT, "examples", "lm_workers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_the_model(example):
    """Against autograd in 64 bits on the bf16 weights.  Differences: every activation, gradient operand and checkpoint is rounded (bf16: 2^-8,
    8 bits: up to one unit, 2^-6 of the block's largest value, 2^-7 on average).  In the 2-norm the roundings of a matrix' entries are
    independent, so that a gradient is off by at most the root of the sum of squares of its chain: two bf16 roundings (activations), one
    checkpoint, two bf16 roundings (dh, dz) and three in the vocabulary's products, 7 * 2^-8 / sqrt(3) and 2^-7 * 3 for a checkpoint whose
    typical value is a third of the largest: 0.03 altogether; a ReLU whose sign falls the other way adds less than that again."""
    sizes = [96, 33, 160]
    w = example.Workers(sizes, 1000, 64, 128, 0.1, 0.9)
    before, after = w.batch()
    loss = w.gradients(before, after)
    w.ops.check()
    flat = w.engine.bf16_shadow().double().clone().requires_grad_(True)
    w1, w2, w3 = w.views(flat)
    at, total = 0, []
    for g, s in enumerate(sizes):
        x = w.embedding[before[at:at + s]].double()
        h = torch.relu(torch.relu(x @ w1[g].T) @ w2[g].T)
        total.append(torch.nn.functional.cross_entropy(h @ w3[g].T, after[at:at + s].long()))
        at += s
    torch.stack(total).sum().backward()
    assert ((loss.double() - torch.stack(total)).abs() <= 0.02 * torch.stack(total)).all()
    for got, want in zip(w.views(w.grads), w.views(flat.grad)):
        assert float((got.double() - want).norm() / want.norm()) <= 0.06
    assert (w.grads[:, sum(n * k for n, k in w.shapes):] == 0).all()


def test_workers_learn_and_agree(example):
    w = example.Workers([512, 256, 512, 256], 512, 128, 256, 0.3, 0.9)
    side = torch.cuda.Stream(priority=-1)
    first = w.round(2, side)
    for _ in range(25):
        last = w.round(4, side)
    w.ops.check()
    w.engine.sync()
    assert float(first.mean()) > 5.0 and float(last.mean()) < 2.5          # log 512 = 6.2, log 4 = 1.4
    x = w.engine.get_params()
    spread = (x - x.mean(0)).norm() / x.norm()
    assert float(spread) < 0.3                                             # the workers' models stay together
