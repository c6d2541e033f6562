"""The calls of a fine-tuning step run together (paper_2305_19982_b200/policy_step.py)."""
import math

import pytest
import torch

from paper_2305_19982_b200.policy_step import PolicyStep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("states", [8, 32])
def test_the_policy_learns_its_task(states):
    """61 answers, 100 steps: chance is 0.016; both kinds of state end far above it."""
    rewards = PolicyStep(vocab=61, states=states).train(100, 2048)
    assert rewards[0] < 0.1 and rewards[-1] > 0.7
    assert all(math.isfinite(r) for r in rewards)


def test_one_step_against_autograd():
    """The gradients that the step's calls produce, against autograd of the loss in fp32 on the same
    bf16 weights.  Logits are rounded to bf16 (2^-9 of |z| <= 8: 1e-2 on p), dlogits and the hidden
    gradient to bf16 once more: 3e-2 relative L2 bounds the inner layer's gradient, and 6e-2 the
    square root of v, which doubles what one rounding of its gradient leaves."""
    p = PolicyStep(vocab=203, dim=64, hidden=96, states=32, seed=3)
    x, y, old, ref, reward = p.rollout(512)
    adv = reward - 0.3 + 0.5 * torch.randn(512, generator=p.gen, device="cuda")
    old = old + 0.01                                   # an off-policy step
    w = torch.full_like(old, 1 / 512)
    emb, inner, head = (t.float().clone().requires_grad_(True) for t in (p.embed_bf, p.inner_bf, p.head_bf))
    logits = (torch.relu(emb[x] @ inner) @ head)[:, :p.vocab]
    logp = torch.log_softmax(logits, 1).gather(1, y[:, None])[:, 0]
    r = torch.exp(logp - old)
    d = ref - logp
    loss = (w * (-torch.minimum(r * adv, r.clamp(0.8, 1.2) * adv) + p.kl_coef * (torch.exp(d) - d - 1))).sum()
    loss.backward()
    before = p.inner.clone()
    p.step(x, y, old, ref, adv, w)
    p.opt.sync_status()
    rel = lambda a, b: float((a.double() - b.double()).norm() / b.double().norm())  # noqa: E731
    assert abs(float(p.stats[0]) - float(loss)) <= 1e-2 * float((w * (adv.abs() + 1)).sum())
    assert rel(p.grads[1], inner.grad) <= 3e-2 and rel(p.grads[0], emb.grad) <= 3e-2
    assert rel(p.head_m[:, :p.vocab] / 0.9, 0.1 * head.grad[:, :p.vocab]) <= 3e-2
    assert rel((p.head_v[:, :p.vocab] / 0.999).sqrt(), (0.001 ** 0.5) * head.grad[:, :p.vocab].abs()) <= 6e-2
    norm = math.sqrt(float(p.grads[0].double().square().sum() + p.grads[1].double().square().sum()))
    assert abs(float(p.norm[0]) - norm) <= 1e-6 * norm
    # the first Adam step moves every weight by lr against the sign of its gradient
    moved = (p.inner - before)[p.grads[1].float().abs() > 1e-6]
    assert torch.allclose(moved.abs(), torch.full_like(moved, p.lr), rtol=2e-2)
    assert torch.equal(p.inner_bf, p.inner.bfloat16()) and torch.equal(p.head_bf, p.head.bfloat16())
    assert not bool(p.head[:, p.vocab:].any())         # the padding columns stay empty


def test_an_infinite_gradient_skips_the_clipped_layers():
    p = PolicyStep(vocab=61, states=8, seed=1)
    x, y, old, ref, reward = p.rollout(64)
    before = [t.clone() for t in (p.embed, p.inner, p.embed_bf)]
    weights = torch.full_like(old, 1 / 64)
    weights[3] = 3e38
    p.step(x, y, old, ref, torch.full_like(old, 10.0), weights)
    assert math.isnan(float(p.norm[1]))
    assert all(torch.equal(a, b) for a, b in zip(before, (p.embed, p.inner, p.embed_bf)))


def test_states_must_be_8_or_32_bits():
    with pytest.raises(ValueError):
        PolicyStep(states=16)
