"""The operators together, as a model with mixtures of experts uses them: its gradients against 64 bits, its scores, its steps."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load(name):
    from paper_1906_12043_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location(name, os.path.join(ROOT, "examples", name + ".py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def exact(m, before, after, chosen):
    """(loss, gradients, logits) by autograd in 64 bits on the bf16 copies, with the experts that were chosen."""
    params = [w.double().requires_grad_(True) for w in m.copies]
    x = m.embedding[before].double()
    for i, experts in enumerate(chosen):
        router, w1, w2 = params[3 * i:3 * i + 3]
        p = torch.softmax(x @ router[0].T, 1).gather(1, experts)
        y = 0
        for j in range(m.top):
            h = torch.relu(torch.einsum("tk,tnk->tn", x, w1[experts[:, j]]))
            y = y + p[:, j:j + 1] * torch.einsum("tn,tkn->tk", h, w2[experts[:, j]])
        x = x + y
    logits = x @ params[-1][0].T
    loss = torch.nn.functional.cross_entropy(logits, after.long())
    loss.backward()
    return loss.detach(), [w.grad for w in params], logits.detach()


@pytest.mark.parametrize("tokens,experts,top,layers", [(300, 8, 2, 2), (77, 16, 4, 1), (1, 8, 1, 2)])
def test_gradients_of_the_model(tokens, experts, top, layers):
    """Every activation and every operand of a gradient is rounded to bf16 once (2^-8 at most, 2^-8 / sqrt 3 in the 2-norm, independent), the checkpoint to 8 bits
    (3 * 2^-7 for typical values a third of the largest).  Along the longest chain (two layers: 4 + 4 activations, 3 in the vocabulary, 4 + 4
    gradients, 2 checkpoints) that is sqrt(19 * 2^-16 / 3 + 2 * 9 * 2^-14) = 0.035; a ReLU whose sign falls the other way adds less than that again.  The router's gradient
    is a difference of terms that are larger than it by up to 3 here (p (1 - p) against p), so that 0.1 is taken for it."""
    m = load("lm_experts").Model(512, 64, 96, experts, top, layers, 1e-3)
    before, after = m.batch(tokens)
    loss, grads = m.gradients(before, after)
    _, _, kept = m.forward(before)
    m.ops.check()
    want_loss, want, _ = exact(m, before, after, [k[2].top_tokens.long() for k in kept])
    assert abs(float(loss) - float(want_loss)) <= 0.02 * float(want_loss)
    for i, (got, g) in enumerate(zip(grads, want)):
        assert got.shape == g.shape
        limit = 0.1 if i % 3 == 0 and i < 3 * layers else 0.07
        if float(g.norm()) > 1e-9:
            assert float((got.double() - g).norm() / g.norm()) <= limit, i
    for k in kept:                                           # the experts are the most probable ones of the logits that were computed
        assert torch.equal(k[2].top_tokens.long(), torch.sort(k[1].float(), dim=1, descending=True, stable=True).indices[:, :top])


def test_steps_and_scores():
    """Both forms of the optimizer run, and the bf16 copies stay those of the parameters; the scores are those of the logits."""
    for bits in (8, 32):
        m = load("lm_experts").Model(512, 64, 96, 8, 2, 2, 1e-3, bits)
        for _ in range(3):
            loss = m.step(*m.batch(200))
        assert torch.isfinite(loss).all() and m.opt.steps == 3
        assert all(torch.equal(p.bfloat16(), c) for p, c in zip(m.params, m.copies))
        before, after = m.batch(150)
        r = m.score(before, after)
        x, whole, _ = m.forward(before)
        logits = m.ops.grouped_forward(x, m.copies[-1], whole).double()
        lp = torch.log_softmax(logits, 1)
        assert (r.logp.double() - lp.gather(1, after.long()[:, None])[:, 0]).abs().max() <= 1e-4
        assert (r.entropy.double() + (lp.exp() * lp).sum(1)).abs().max() <= 1e-4
        assert torch.equal(r.top_tokens.long(), torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :4])
        m.ops.check()


def test_a_captured_step_is_the_step():
    """Forward, backward and update in one graph: the same bits as the calls, step after step."""
    made = load("lm_experts")
    a, b = (made.Model(512, 64, 96, 8, 2, 2, 1e-3) for _ in range(2))
    before, after = a.batch(128)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.gradients(before, after)                           # (nothing is updated)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        loss = a.step(before, after)
    for _ in range(3):
        x, y = b.batch(128)
        before.copy_(x)
        after.copy_(y)
        graph.replay()
        assert torch.equal(loss, b.step(x, y))
        assert all(torch.equal(p, q) for p, q in zip(a.params, b.params))
    assert a.opt.steps == b.opt.steps == 3
    a.ops.check()


@pytest.mark.parametrize("bits", [8, 32])
def test_workers_with_adamw(bits):
    """The workers of the other example, with AdamW local steps in rounds of Algorithm 1."""
    made = load("lm_workers")
    w = made.Workers([96, 33, 160], 1000, 64, 128, 1e-3, 0.9, adamw_bits=bits)
    side = torch.cuda.Stream(priority=-1)
    for _ in range(2):
        losses = w.round(3, side)
    w.ops.check()
    w.engine.sync()
    assert torch.isfinite(losses).all() and w.opt.steps == 6 and w.engine.step_count == 6
    x = w.engine.get_params()
    assert torch.isfinite(x).all() and torch.equal(w.engine.bf16_shadow(), x.bfloat16())
