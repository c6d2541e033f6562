"""The calls of a distillation step run together (paper_2305_19982_b200/distill_step.py)."""
import pytest
import torch

from paper_2305_19982_b200.distill_step import DistillStep

pytestmark = pytest.mark.gpu


def _loss(p, w, x, values, ids, lse):
    """The same loss in fp32 by torch operations; `w` as p.w, differentiable.  The hidden layer's input is rounded
    to bf16 as the step does (a sum near 0 whose sign flipped would switch a whole gradient on or off)."""
    e = torch.where((x >= 0)[:, None], w[0][x.clamp(min=0)], 0.0)
    norm = torch.nn.functional.layer_norm
    n = norm(e, e.shape[1:], w[1], w[2])
    h = torch.relu((n + (n.bfloat16().float() - n).detach()) @ w[3])
    logq = torch.log_softmax((norm(h, h.shape[1:], w[4], w[5]) @ w[6])[:, :p.vocab], 1).gather(1, ids)
    logp = values.float() - lse[:, None]
    return ((logp.exp() * (logp - logq)).sum(1) * (x >= 0)).sum() / x.numel()


@pytest.mark.parametrize("vocab,dim,hidden,top,tokens", [(203, 64, 96, 16, 512), (1003, 128, 256, 1, 700), (5001, 40, 72, 128, 333)])
def test_one_step_against_autograd(vocab, dim, hidden, top, tokens):
    """The moments after a step of two micro-batches against those that autograd's gradients give in fp32, from the same
    bf16 weights.  On the way to the table's gradient stand eight roundings to bf16 (hidden row, normed hidden row, logits,
    dlogits, and the gradients of the two norms' outputs and inputs), each at most 2^-8 of its tensor and passed on about
    once: 8*2^-8 = 3.2e-2 relative L2 on a gradient, and twice that on the square root of v, whose own rounding
    doubles there."""
    p = DistillStep(vocab=vocab, dim=dim, hidden=hidden, top=top, seed=3)
    for i in (1, 4):     # norms with weights and biases of their own
        p.w[i].add_(0.2 * torch.randn(p.w[i].shape, generator=p.gen, device="cuda"))
        p.w[i + 1].add_(0.2 * torch.randn(p.w[i].shape, generator=p.gen, device="cuda"))
    batches = [p.batch(tokens, padding=0.2) for _ in range(2)]
    before = [w.clone() for w in p.w]
    leaves = [p.copies.get(i, w).float().clone().requires_grad_(True) for i, w in enumerate(p.w)]
    losses = [_loss(p, leaves, *b) for b in batches]
    grads = [torch.autograd.grad(loss, leaves) for loss in losses]
    p.step(batches)
    p.opt.sync_status()
    rel = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())  # noqa: E731
    assert abs(float(p.stats[0]) - float(losses[1].detach())) <= 2e-2 * float(losses[1].detach().abs()) + 1e-3
    for i, (g0, g1) in enumerate(zip(*grads)):
        assert rel(p.m[i] / 0.9, 0.1 * (g0 + g1) / 2) <= 3.2e-2, i
        assert rel((p.v[i] / 0.999).sqrt(), (0.001 * (g0 * g0 + g1 * g1) / 4).sqrt()) <= 6.4e-2, i
    # rows of the table whose token did not occur, or only as padding, stay
    seen = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    for b in batches:
        seen[b[0][b[0] >= 0]] = True
    assert torch.equal(p.w[0][~seen], before[0][~seen]) and not bool(p.m[0][~seen].any())
    assert not bool(p.w[6][:, vocab:].any())           # the padding columns stay empty
    assert all(torch.equal(c, p.w[i].bfloat16()) for i, c in p.copies.items())
    assert all(not torch.equal(a, b) for a, b in zip(before, p.w))


def test_a_step_repeats_exactly():
    runs = []
    for _ in range(2):
        p = DistillStep(vocab=307, seed=5)
        p.train(3, 600)
        runs.append(p.w + p.m + p.v + [p.stats])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_micro_batches_in_graphs():
    """Two captured micro-batches of different lengths, replayed in either order and between eager ones."""
    p = DistillStep(vocab=307, seed=6)
    batches = [p.batch(n, padding=0.1) for n in (600, 1100, 257)]
    side = torch.cuda.Stream()
    p.opt.begin_minibatch(4)
    for b in batches:
        p.micro_batch(*b)

    def moments(calls):
        for t in p.m + p.v:
            t.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for call in calls:
                call()
        torch.cuda.synchronize()
        return [t.clone() for t in p.m + p.v]

    graphs = []
    for b in batches[:2]:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            p.micro_batch(*b)
        graphs.append(g)
    eager = [lambda b=b: p.micro_batch(*b) for b in batches]
    for order in ((0, 1), (1, 2, 0), (2, 1, 0, 1)):
        want = moments([eager[i] for i in order])
        got = moments([graphs[i].replay if i < 2 else eager[i] for i in order])
        assert all(torch.equal(a, b) for a, b in zip(want, got)), order
    p.opt.sync_status()
