"""A step with a gradient that is not finite leaves the whole model as it was (policy_step.py)."""
import math

import pytest
import torch

from paper_2305_19982_b200.policy_step import PolicyStep

pytestmark = pytest.mark.gpu


def _model(p):
    return [p.embed, p.inner, p.head, p.embed_bf, p.inner_bf, p.head_bf, p.head_m, p.head_v]


@pytest.mark.parametrize("states", [8, 32])
@pytest.mark.parametrize("weight", [3e38, math.inf, math.nan, 1e30])
def test_a_step_that_is_not_finite_is_skipped_by_every_layer(states, weight):
    """1e30: the loss's gradient is finite, its square, which v holds, is not.  A step before gives the
    moments values; one after learns again."""
    p = PolicyStep(vocab=61, states=states, seed=1)
    x, y, old, ref, reward = p.rollout(64)
    adv, weights = torch.full_like(old, 10.0), torch.full_like(old, 1 / 64)
    p.step(x, y, old, ref, adv, weights)
    before = [t.clone() for t in _model(p)]
    bad = weights.clone()
    bad[3] = weight
    p.step(x, y, old, ref, adv, bad)
    assert math.isnan(float(p.norm[1]))
    assert all(torch.equal(a, b) for a, b in zip(before, _model(p)))
    p.step(x, y, old, ref, adv, weights)
    assert all(math.isfinite(float(s)) for s in p.stats)
    assert all(bool(torch.isfinite(t.float()).all()) for t in _model(p))
    assert not any(torch.equal(a, b) for a, b in zip(before, _model(p)))
    p.opt.sync_status()


def test_a_step_that_only_the_output_layer_cannot_take_is_skipped_too():
    """The layers in front see finite gradients (the output layer's weights pass on little); the output
    layer's own would be infinite in v."""
    p = PolicyStep(vocab=61, states=32, seed=2)
    p.head_bf.mul_(1e-30)
    x, y, old, ref, reward = p.rollout(64)
    before = [t.clone() for t in _model(p)]
    p.step(x, y, old, ref, torch.full_like(old, 10.0), torch.full_like(old, 1e22))
    assert math.isfinite(float(p.norm[0]))
    assert all(torch.equal(a, b) for a, b in zip(before, _model(p)))
