"""The policy loss at the ends of its values: policies that hardly differ, ratios that overflow.

Tolerances.  d = ref - logp is exact here (both are close, or far from rounding).  A KL term is one
series of 8 products (8*2^-24), or exp(d) - 1 - d at |d| >= 1/2: 2^-23 of exp(d) against at least 0.106,
1.2e-6.  KL = 2e-6 relative bounds both, the terms being positive also their sum.  The gradient's
factor exp(d) - 1 carries the same, p its 1e-5 as everywhere: GRAD = 4e-5 of unit*(p + [j = target])."""
import math

import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama

pytestmark = pytest.mark.gpu
KL, GRAD = 2e-6, 4e-5
SHAPES = [(40, 500), (33, 9_001), (20, 50_257), (6, 131_072), (3, 460_001)]   # a warp to a row .. rows read twice


def _rows(T, V, seed):
    x = wl.normal((T, V), 1.0, torch.float32, seed).cuda()
    targets = (torch.arange(T, device="cuda") * 7919) % V
    logp = torch.empty(T, device="cuda")
    zero, stats = torch.zeros(T, device="cuda"), torch.empty(4, device="cuda")
    opt = adama.AdamA()
    opt.policy_loss(x, targets, zero, zero, torch.ones(T, device="cuda"), None, stats, logp=logp)
    return opt, x, targets, logp


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("size", [1e-5, 1e-4, 3e-4, 1e-3, 1e-2, 0.1, 0.45, 0.55, 2.0, 20.0])
def test_kl_of_policies_that_hardly_differ(T, V, size):
    """One row's logp against a reference `size` away, both signs; the advantage is 0, so that the loss and
    the gradient are the KL term's alone."""
    opt, x, targets, logp = _rows(T, V, 3)
    sign = 1.0 - 2.0 * (torch.arange(T, device="cuda") % 2)
    ref = logp + sign * size
    d = ref.double() - logp.double()
    w = torch.rand(T, generator=torch.Generator().manual_seed(1)).cuda() + 0.5
    grad, stats = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")
    opt.policy_loss(x, targets, logp, torch.zeros(T, device="cuda"), w, grad, stats, ref_logp=ref, kl_coef=1.0)
    e1 = torch.expm1(d)
    # (expm1(d) - d in 64 bits cancels to 2^-53/(d/2): 5e-11 at 1e-5)
    want = float((w.double() * (e1 - d)).sum())
    assert abs(float(stats[2]) - want) <= KL * want
    assert abs(float(stats[0]) - want) <= KL * want and float(stats[1]) == 0.0
    unit = w.double() * -e1
    for i in range(T):
        p = torch.softmax(x[i].double(), 0)
        hot = torch.zeros_like(p)
        hot[targets[i]] = 1
        err = (grad[i].double() - unit[i] * (hot - p)).abs()
        assert bool((err <= GRAD * unit[i].abs() * (p + hot) + 1e-30).all())


def test_equal_policies_have_no_kl_and_no_gradient():
    opt, x, targets, logp = _rows(40, 500, 4)
    grad, stats = torch.full((40, 500), 5.0, device="cuda"), torch.empty(4, device="cuda")
    opt.policy_loss(x, targets, logp, torch.zeros(40, device="cuda"), torch.ones(40, device="cuda"), grad, stats,
                    ref_logp=logp, kl_coef=1.0)
    assert stats.tolist() == [0.0] * 4 and not bool(grad.any())


@pytest.mark.parametrize("T,V", SHAPES)
def test_kl_that_is_only_watched_does_not_reach_the_loss(T, V):
    """kl_coef 0 with a reference that is far away, so that exp(ref - logp) overflows: the KL is infinite,
    loss and gradient are those without a reference."""
    opt, x, targets, logp = _rows(T, V, 5)
    old, one = logp - 0.1, torch.ones(T, device="cuda")
    grads, stats = [torch.empty(T, V, device="cuda") for _ in range(2)], [torch.empty(4, device="cuda") for _ in range(2)]
    opt.policy_loss(x, targets, old, one, one, grads[0], stats[0])
    opt.policy_loss(x, targets, old, one, one, grads[1], stats[1], ref_logp=logp + 100, kl_coef=0.0)
    assert torch.equal(grads[0], grads[1]) and torch.equal(stats[0][:2], stats[1][:2])
    assert float(stats[1][2]) == math.inf and math.isfinite(float(stats[1][0]))


@pytest.mark.parametrize("T,V", SHAPES)
def test_no_advantage_no_loss_however_large_the_ratio(T, V):
    """exp(logp - old) = exp(100) overflows fp32; times an advantage of 0 it is 0.  A NaN ratio stays visible."""
    opt, x, targets, logp = _rows(T, V, 6)
    grad, stats = torch.full((T, V), 5.0, device="cuda"), torch.empty(4, device="cuda")
    zero, one = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    opt.policy_loss(x, targets, logp - 100, zero, one, grad, stats)
    assert stats.tolist() == [0.0] * 4 and not bool(grad.any())
    opt.policy_loss(x, targets, torch.full_like(logp, math.nan), zero, one, grad, stats)
    assert math.isnan(float(stats[0])) and bool(torch.isnan(grad).all())


def test_a_scale_that_overflows_fp32_is_refused():
    """2.5e38*log2(e), the factor of the exponentials, is beyond fp32."""
    opt, x, targets, logp = _rows(4, 50, 7)
    launches, one, stats = opt.launch_count, torch.ones(4, device="cuda"), torch.empty(4, device="cuda")
    for scale in (2.5e38, 1e39, 1e300):
        for call in (lambda: opt.token_logprobs(x, targets, logp, logit_scale=scale),
                     lambda: opt.policy_loss(x, targets, logp, one, one, None, stats, logit_scale=scale)):
            with pytest.raises(adama.AdamAError) as e:
                call()
            assert e.value.status == adama.Status.ERR_INVALID_ARG and "logit_scale" in str(e.value)
    assert opt.launch_count == launches
