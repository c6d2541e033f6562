"""Token log-probabilities (adama_token_logprobs) and the clipped policy loss with its gradient
(adama_policy_loss) against the definitions in 64 bits.

Tolerances.  With |z - lse| <= 60 and rows of at most 2^17 elements: each exp(z - ref) carries
2^-22 (the exponential) + 60*2^-24 (its argument) and a sum of V terms over the threads and warps at
most (V/512 + 40)*2^-24 relative: 2.4e-7 + 3.6e-6 + (1.6e-5 at 2^17, worst case; the roundings'
random walk stays under 1e-6).  LOGP = 1e-5 absolute bounds logp, lse and entropy/|z|; a factor
exp(logp - old) turns that into 1e-5 relative; p adds another 1e-5: GRAD = 4e-5 of unit*(p + [j =
target]), plus half a last place of the output's type.  unit is w*s times the SUM of the magnitudes
of the two terms of dloss/dlogp: each carries the relative error, and they may cancel."""
import math

import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu
LOGP, GRAD = 1e-5, 4e-5
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def _logits(T, V, dtype, seed, ld=None, offset=0, std=3.0):
    """[T, V] logits with pitch ld at `offset` elements past an aligned start, sentinels around."""
    ld = V if ld is None else ld
    buf = torch.full((offset + T * ld + 64,), 777.0, dtype=dtype, device="cuda")
    view = buf[offset:offset + T * ld].view(T, ld)[:, :V]
    view.copy_(wl.normal((T, V), std, torch.float32, seed))
    return buf, view


def _reference(x, targets, scale):
    """lse, logp, entropy, p in float64."""
    z = x.double().cpu() * scale
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    t = targets.cpu().clamp(min=0)
    return lse, z.gather(1, t[:, None])[:, 0] - lse, -torch.xlogy(p, p).sum(1), p


SHAPES = [(1, 1), (1, 2), (3, 7), (2, 8), (5, 100), (4, 1000), (3, 4099), (2, 50257), (300, 513), (1, 131072), (700, 33), (2, 160_001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("pitch,offset,scale", [(0, 0, 1.0), (5, 3, 1.25), (24, 8, 0.5)])
def test_token_logprobs(T, V, dtype, pitch, offset, scale):
    opt = adama.AdamA()
    buf, x = _logits(T, V, dtype, T + V, V + pitch, offset)
    targets = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(V)).cuda()
    logp, lse, ent = (torch.full((T,), -7.0, device="cuda") for _ in range(3))
    opt.token_logprobs(x, targets, logp, lse=lse, entropy=ent, logit_scale=scale)
    rl, rp, re, _ = _reference(x, targets, scale)
    assert float((lse.cpu().double() - rl).abs().max()) <= LOGP
    assert float((logp.cpu().double() - rp).abs().max()) <= LOGP
    assert float((ent.cpu().double() - re).abs().max()) <= LOGP * 10
    only = torch.empty(T, device="cuda")
    opt.token_logprobs(x, targets, only, logit_scale=scale)          # lse and entropy left out
    assert torch.equal(only, logp)
    opt.sync_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(20, 9001), (100, 26_001), (300, 9001), (300, 30_011), (470, 26_001), (760, 26_001), (1600, 26_001)])
def test_token_logprobs_at_every_number_of_warps_to_a_row(T, V, dtype):
    opt = adama.AdamA()
    buf, x = _logits(T, V, dtype, T + V, V + 1, 1)
    targets = torch.randint(-1, V, (T,), generator=torch.Generator().manual_seed(V)).cuda()
    logp, lse, ent = (torch.full((T,), -7.0, device="cuda") for _ in range(3))
    opt.token_logprobs(x, targets, logp, lse=lse, entropy=ent)
    live = targets.cpu() >= 0
    rl, rp, re, _ = (r[live] for r in _reference(x, targets, 1.0))
    assert float((lse.cpu().double()[live] - rl).abs().max()) <= LOGP
    assert float((logp.cpu().double()[live] - rp).abs().max()) <= LOGP
    assert float((ent.cpu().double()[live] - re).abs().max()) <= LOGP * 10
    assert not (~live).any() or float(logp.cpu()[~live].abs().max()) == 0.0
    opt.sync_status()


def test_token_logprobs_of_rows_with_infinite_entries():
    opt = adama.AdamA()
    T, V = 6, 3001
    _, x = _logits(T, V, torch.float32, 5)
    x[0, :2900] = -math.inf                       # whole threads and warps see nothing but -inf
    x[1, 1:] = -math.inf                          # one entry left: probability 1
    x[2, :] = -math.inf                           # nothing left
    x[3, 17] = math.nan
    x[4, 5:] = torch.finfo(torch.float32).min     # the type's lowest value instead of -inf
    targets = torch.tensor([2950, 0, 1, 1, 2, 100]).cuda()
    x[5, 100] = -math.inf                         # the target itself is masked
    logp, lse, ent = (torch.empty(T, device="cuda") for _ in range(3))
    opt.token_logprobs(x, targets, logp, lse=lse, entropy=ent)
    rl, rp, re, _ = _reference(x, targets, 1.0)
    for i in (0, 1, 4):
        assert abs(float(lse[i]) - float(rl[i])) <= LOGP and abs(float(logp[i]) - float(rp[i])) <= LOGP
        assert abs(float(ent[i]) - float(re[i])) <= 10 * LOGP
    assert float(logp[1]) == 0.0
    assert float(lse[2]) == -math.inf and math.isnan(float(logp[2]))
    assert math.isnan(float(logp[3])) and math.isnan(float(lse[3]))
    assert float(logp[5]) == -math.inf


def test_a_common_offset_of_the_logits_costs_no_precision():
    """Adding 4096 to every logit (exact in fp32 for these) leaves logp and the gradient alone: the
    differences from the largest logit are what is computed with."""
    opt = adama.AdamA()
    T, V = 4, 5000
    x = (torch.randint(-200, 200, (T, V), generator=torch.Generator().manual_seed(1)) / 64.0).cuda()
    targets = torch.arange(T).cuda()
    out = []
    for shift in (0.0, 4096.0):
        logp, d, stats = torch.empty(T, device="cuda"), torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")
        one = torch.ones(T, device="cuda")
        opt.token_logprobs(x + shift, targets, logp)
        opt.policy_loss(x + shift, targets, logp, one, one, d, stats)
        out.append((logp, d))
    assert float((out[0][0] - out[1][0]).abs().max()) <= LOGP
    assert float((out[0][1] - out[1][1]).abs().max()) <= GRAD * float(out[0][1].abs().max())


def test_negative_targets_are_ignored_and_large_ones_reported():
    opt = adama.AdamA()
    _, x = _logits(4, 50, torch.float32, 3)
    targets = torch.tensor([-100, 3, 50, 1 << 40]).cuda()
    logp, lse = torch.full((4,), 9.0, device="cuda"), torch.full((4,), 9.0, device="cuda")
    opt.token_logprobs(x, targets, logp, lse=lse)
    assert float(logp[0]) == 0 and float(lse[0]) == 0 and math.isfinite(float(logp[1]))
    assert torch.isnan(logp[2:]).all() and torch.isfinite(lse[2:]).all()
    with pytest.raises(adama.AdamAError) as e:
        opt.sync_status()
    assert e.value.status == Status.ERR_INVALID_ARG and "target" in str(e.value)
    opt.sync_status()                             # cleared by the report


def _policy_reference(x, targets, old, adv, weights, ref, cl, ch, beta, scale):
    """Loss terms and gradient in float64 (the gradient from autograd of the loss as written)."""
    x64 = x.double().cpu().requires_grad_(True)
    z = x64 * scale
    logp = torch.log_softmax(z, 1).gather(1, targets.cpu().clamp(min=0)[:, None])[:, 0]
    r = torch.exp(logp - old.double().cpu())
    A, w = adv.double().cpu(), weights.double().cpu()
    w = torch.where(targets.cpu() >= 0, w, 0.0)
    clipped = torch.clamp(r, 1 - cl, 1 + ch) * A
    pg = -torch.minimum(r * A, clipped)
    kl = torch.zeros_like(pg)
    if ref is not None:
        d = ref.double().cpu() - logp
        kl = torch.exp(d) - d - 1
    loss = (w * (pg + beta * kl)).sum()
    loss.backward()
    cut = (r * A > clipped).double()
    size = torch.where(r * A > clipped, 0.0, (r * A).abs())
    if ref is not None:
        size = size + abs(beta) * (1 + torch.exp(d))
    terms = [float(v.detach()) for v in (loss, (w * pg).sum(), (w * kl).sum(), (w * cut).sum())]
    return terms, x64.grad, logp.detach(), (w * scale * size).detach()[:, None]


def _policy_inputs(T, V, dtype, seed, ld=None, offset=0, scale=1.0, with_ref=True):
    gen = torch.Generator().manual_seed(seed)
    buf, x = _logits(T, V, dtype, seed, ld, offset, std=2.0)
    targets = torch.randint(0, V, (T,), generator=gen)
    logp = torch.log_softmax(x.double().cpu() * scale, 1).gather(1, targets[:, None])[:, 0]
    # log ratios on a grid that keeps 3e-4 away from the clip boundaries
    step = lambda s: ((torch.randn(T, generator=gen) * s * 512).round() + 0.5) / 512  # noqa: E731
    old = (logp - step(0.2)).float().cuda()
    ref = (logp - step(0.4)).float().cuda() if with_ref else None
    adv = torch.randn(T, generator=gen).cuda()
    weights = torch.rand(T, generator=gen)
    if T > 2:
        weights[::3] = 0
        targets[1] = -1
    return buf, x, targets.cuda(), old, ref, adv, weights.cuda()


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16),
                                       (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("pitch,offset,scale,ref", [(0, 0, 1.0, True), (3, 1, 1.25, False)])
def test_policy_loss_and_gradient(T, V, dtype, out, pitch, offset, scale, ref):
    opt = adama.AdamA()
    buf, x, targets, old, ref, adv, weights = _policy_inputs(T, V, dtype, 7 * T + V, V + pitch, offset, scale, ref)
    keep = buf.clone()
    dbuf, d = _logits(T, V, out, 1, V + pitch, offset)
    stats, logp = torch.empty(4, device="cuda"), torch.full((T,), 5.0, device="cuda")
    opt.policy_loss(x, targets, old, adv, weights, d, stats, ref_logp=ref, logp=logp, clip_low=0.2, clip_high=0.28,
                    kl_coef=0.1, logit_scale=scale)
    opt.sync_status()
    terms, grad, rlogp, unit = _policy_reference(x, targets, old, adv, weights, ref, 0.2, 0.28, 0.1, scale)
    assert torch.equal(buf, keep)                                       # logits are only read
    live = (weights != 0).cpu() & (targets.cpu() >= 0)
    assert float((logp.cpu().double() - torch.where(live, rlogp, 0.0)).abs().max()) <= LOGP
    # each term: relative error 1e-5 through the ratio, weights and |A| of order one
    size = float((weights.double().cpu() * (adv.double().abs().cpu() * 4 + 2)).sum())
    for got, want in zip(stats.tolist(), terms):
        assert abs(got - want) <= 2 * LOGP * size + 1e-6
    p = torch.softmax(x.double().cpu() * scale, 1)
    hot = torch.zeros(T, V, dtype=torch.float64).scatter_(1, targets.cpu().clamp(min=0)[:, None], 1.0)
    bound = GRAD * unit * (p + hot) + HALF_ULP[out] * grad.abs() + 1e-30
    err = (d.double().cpu() - grad).abs()
    assert bool((err[live] <= bound[live]).all()), float((err - bound)[live].max())
    assert not bool(d.cpu()[~live].any())
    tail = dbuf[offset:offset + T * (V + pitch)].view(T, V + pitch)[:, V:]
    assert bool((tail == 777.0).all()) and bool((dbuf[:offset] == 777.0).all()) and bool((dbuf[offset + T * (V + pitch):] == 777.0).all())
    # the same pass writing over the logits, and the one without a gradient
    second, third = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    kw = dict(ref_logp=ref, clip_low=0.2, clip_high=0.28, kl_coef=0.1, logit_scale=scale)
    opt.policy_loss(x, targets, old, adv, weights, None, third, **kw)
    assert torch.equal(stats, third)
    if dtype == out:
        opt.policy_loss(x, targets, old, adv, weights, x, second, **kw)
        assert torch.equal(stats, second) and torch.equal(x, d)


LONG = [(1300, 5_003), (700, 9_001), (400, 20_001), (160, 16_385), (150, 51_200), (150, 51_203), (160, 57_345), (152, 65_537), (80, 131_073), (2, 229_381), (2, 458_760), (3, 459_001), (2, 460_001), (1, 920_003)]


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("T,V", LONG)
@pytest.mark.parametrize("pitch,out_pitch", [(0, 0), (1, 7)])
def test_policy_loss_of_long_rows(T, V, dtype, out, pitch, out_pitch):
    """Rows of one CTA, of a cluster, and longer than a cluster holds; with the gradient's rows
    aligned like the logits' and otherwise.  Same bounds as above; the reference in 64 bits is
    evaluated on the GPU."""
    opt = adama.AdamA()
    gen = torch.Generator(device="cuda").manual_seed(T + V)
    rows = torch.randn(T, V + pitch, generator=gen, device="cuda").to(dtype).mul_(2)
    x = rows[:, :V]
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    targets[:4 if T > 4 else 1] = torch.tensor([0, V - 1, V // 2, 7], device="cuda")[:4 if T > 4 else 1]
    logp = torch.stack([r.double()[t] - torch.logsumexp(r.double(), 0) for r, t in zip(x, targets)])
    step = lambda s: ((torch.randn(T, generator=gen, device="cuda") * s * 512).round() + 0.5) / 512  # noqa: E731
    old, ref = (logp - step(0.2)).float(), (logp - step(0.4)).float()
    adv, weights = torch.randn(T, generator=gen, device="cuda"), torch.rand(T, generator=gen, device="cuda")
    weights[2::5] = 0
    whole = torch.full((T, V + out_pitch), 777.0, dtype=out, device="cuda")
    d, stats, got = whole[:, :V], torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.policy_loss(x, targets, old, adv, weights, d, stats, ref_logp=ref, logp=got, kl_coef=0.1)
    opt.sync_status()
    r, dd = torch.exp(logp - old.double()), ref.double() - logp
    A, w = adv.double(), weights.double()
    clipped = r.clamp(0.8, 1.2) * A
    cut = r * A > clipped
    slope = torch.where(cut, 0.0, -r * A) + 0.1 * (1 - torch.exp(dd))
    size = (torch.where(cut, 0.0, (r * A).abs()) + 0.1 * (1 + torch.exp(dd))) * w
    assert float((got.double() - torch.where(w != 0, logp, 0.0)).abs().max()) <= LOGP
    pg, kl = -torch.minimum(r * A, clipped), torch.exp(dd) - dd - 1
    for value, terms in zip(stats.tolist(), (pg + 0.1 * kl, pg, kl, cut.double())):
        assert abs(value - float((w * terms).sum())) <= 2 * LOGP * float((w * (4 * A.abs() + 2)).sum()) + 1e-6
    for i in range(T):
        p = torch.softmax(x[i].double(), 0)
        grad = -p
        grad[targets[i]] += 1
        grad = grad * (w[i] * slope[i])
        p[targets[i]] += 1
        bound = GRAD * size[i] * p + HALF_ULP[out] * grad.abs() + 1e-30
        err = (d[i].double() - grad).abs()
        assert bool((err <= bound).all()), (i, float((err - bound).max()))
        if float(w[i]) == 0:
            assert not bool(d[i].any())
    assert bool((whole[:, V:] == 777.0).all())
    if dtype == out and pitch == 0:
        second = torch.empty(4, device="cuda")
        opt.policy_loss(x, targets, old, adv, weights, x, second, ref_logp=ref, kl_coef=0.1)
        assert torch.equal(second, stats) and torch.equal(x, d)


def test_gradient_against_differences():
    """Directional derivative: (loss(x + h*u) - loss(x - h*u))/2h with h = 1/64 against <dlogits, u>;
    u has unit entries, the truncation is h^2/6 of a third derivative of order |unit| and the loss's
    rounding 1e-6/h: 1e-3 of the gradient's scale bounds both."""
    opt = adama.AdamA()
    T, V, h = 5, 37, 1 / 64
    _, x, targets, old, ref, adv, weights = _policy_inputs(T, V, torch.float32, 99)
    old = old - 0.01
    kw = dict(ref_logp=ref, clip_low=0.5, clip_high=0.9, kl_coef=0.3)
    d, stats = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")
    opt.policy_loss(x, targets, old, adv, weights, d, stats, **kw)
    gen = torch.Generator().manual_seed(1)
    for _ in range(6):
        u = (torch.randint(0, 2, (T, V), generator=gen) * 2.0 - 1).cuda()
        ends = []
        for sign in (1, -1):
            opt.policy_loss(x + sign * h * u, targets, old, adv, weights, None, stats, **kw)
            ends.append(float(stats[0]))
        diff = (ends[0] - ends[1]) / (2 * h)
        assert abs(diff - float((d * u).sum())) <= 1e-3 * float(d.abs().sum()) + 1e-4


def test_the_clip_cuts_the_gradient_where_it_should():
    """Four rows, ratio above and below the range, advantage of both signs: the policy gradient is
    zero exactly where min picks the clamped product."""
    opt = adama.AdamA()
    V = 64
    _, x = _logits(4, V, torch.float32, 8)
    targets = torch.zeros(4, dtype=torch.int64, device="cuda")
    logp = torch.empty(4, device="cuda")
    opt.token_logprobs(x, targets, logp)
    old = logp - torch.tensor([0.5, 0.5, -0.5, -0.5], device="cuda")
    adv = torch.tensor([1.0, -1.0, 1.0, -1.0], device="cuda")
    d, stats, one = torch.empty(4, V, device="cuda"), torch.empty(4, device="cuda"), torch.ones(4, device="cuda")
    opt.policy_loss(x, targets, old, adv, one, d, stats)
    assert [bool(r.any()) for r in d] == [False, True, True, False]
    assert float(stats[3]) == 2.0
    want = -(1.2 - math.exp(0.5) + math.exp(-0.5) - 0.8)
    assert abs(float(stats[0]) - want) <= 1e-5 and float(stats[0]) == float(stats[1]) and float(stats[2]) == 0.0


def test_rows_with_infinite_entries_and_masked_rows_of_nan():
    opt = adama.AdamA()
    T, V = 4, 2050
    _, x, targets, old, ref, adv, weights = _policy_inputs(T, V, torch.bfloat16, 11)
    weights.copy_(torch.tensor([0.5, 0.25, 0.0, 0.125]))
    targets.copy_(torch.tensor([3, 2049, 5, 7]))
    x[0, 100:] = -math.inf
    x[1, :2048] = torch.finfo(torch.bfloat16).min
    x[2, :] = math.nan                             # weight 0: not looked at
    x[3, 8:] = -math.inf
    d, stats = torch.full((T, V), 9.0, dtype=torch.bfloat16, device="cuda"), torch.empty(4, device="cuda")
    logp = torch.empty(T, device="cuda")
    opt.token_logprobs(x, torch.where(weights > 0, targets, -1), logp)
    old = logp - 0.1
    opt.policy_loss(x, targets, old, adv, weights, d, stats, ref_logp=logp - 0.3, kl_coef=0.5)
    assert torch.isfinite(d.float()).all() and torch.isfinite(stats).all()
    assert not bool(d[2].any()) and not bool(d[0, 100:].any()) and not bool(d[1, :2048].any()) and not bool(d[3, 8:].any())
    for i in (0, 1, 3):                            # a gradient of a softmax sums to zero
        assert abs(float(d[i].double().sum())) <= 3e-2 * float(d[i].double().abs().sum())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V", [(3, 100), (2, 3001), (2, 40_003), (200, 20_001), (2, 131_074)])
def test_rows_at_the_lowest_value_are_uniform(T, V, dtype):
    """A row that a mask has set to the type's lowest value throughout is a uniform one."""
    opt = adama.AdamA()
    x = torch.full((T, V), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    targets = torch.arange(T, device="cuda") % V
    logp, lse, ent = (torch.empty(T, device="cuda") for _ in range(3))
    opt.token_logprobs(x, targets, logp, lse=lse, entropy=ent)
    assert float((logp + math.log(V)).abs().max()) <= LOGP and float((ent - math.log(V)).abs().max()) <= 10 * LOGP
    one, d, stats = torch.ones(T, device="cuda"), torch.empty(T, V, dtype=dtype, device="cuda"), torch.empty(4, device="cuda")
    opt.policy_loss(x, targets, logp, one, one, d, stats)
    want = torch.full((T, V), 1.0 / V, dtype=torch.float64, device="cuda")
    want[torch.arange(T, device="cuda"), targets] -= 1
    assert bool(((d.double() - want).abs() <= GRAD * want.abs() + HALF_ULP[dtype] * want.abs()).all())


def test_large_logits_saturate_without_overflow():
    opt = adama.AdamA()
    T, V = 3, 300
    x = torch.full((T, V), -1e30, device="cuda")
    x[:, 7] = 3e4
    x[2, 9] = 3e4
    targets = torch.tensor([7, 3, 9]).cuda()
    logp, ent = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    opt.token_logprobs(x, targets, logp, entropy=ent)
    assert float(logp[0]) == 0.0 and abs(float(logp[2]) + math.log(2)) <= LOGP and float(logp[1]) < -1e29
    assert float(ent[0]) == 0.0 and abs(float(ent[2]) - math.log(2)) <= LOGP


def test_run_twice_is_deterministic_and_streams_do_not_share_scratch():
    opt = adama.AdamA()
    T, V = 1000, 1031
    _, x, targets, old, ref, adv, weights = _policy_inputs(T, V, torch.bfloat16, 21)
    outs, streams = [], [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            d, stats = torch.empty(T, V, dtype=torch.bfloat16, device="cuda"), torch.empty(4, device="cuda")
            for _ in range(3):
                opt.policy_loss(x, targets, old, adv, weights, d, stats, ref_logp=ref, kl_coef=0.1)
            outs.append((d, stats))
    torch.cuda.synchronize()
    for d, stats in outs[1:]:
        assert torch.equal(d, outs[0][0]) and torch.equal(stats, outs[0][1])


def test_offsets_beyond_32_bits():
    """Rows that begin past 2^32 bytes and 2^31 elements: a pitch of 2^22 elements, 1030 rows."""
    T, V, ld = 1030, 1001, 1 << 22
    opt = adama.AdamA()
    buf = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda")
    x = buf.view(T, ld)[:, :V]
    x.copy_(wl.normal((T, V), 2.0, torch.float32, 3))
    targets = torch.arange(T).cuda() % V
    logp, small = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    opt.token_logprobs(x, targets, logp)
    dense = x.contiguous()
    opt.token_logprobs(dense, targets, small)
    assert float((logp - small).abs().max()) <= LOGP
    one, s1, s2 = torch.ones(T, device="cuda") / T, torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    d = torch.empty_like(dense)
    opt.policy_loss(dense, targets, small, one, one, d, s1)
    opt.policy_loss(x, targets, small, one, one, x, s2)
    assert float((x.float() - d.float()).abs().max()) <= 2.0 ** -7 * float(d.float().abs().max())


def test_policy_refusals():
    opt = adama.AdamA()
    T, V = 4, 50
    _, x, targets, old, ref, adv, weights = _policy_inputs(T, V, torch.float32, 1)
    d, stats, logp = torch.zeros(T, V, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda")

    def err(fn, *a, **k):
        with pytest.raises(adama.AdamAError) as e:
            fn(*a, **k)
        return e.value.status

    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-1.0), dict(kl_coef=math.inf),
               dict(logit_scale=0.0), dict(logit_scale=math.nan)):
        assert err(opt.policy_loss, x, targets, old, adv, weights, d, stats, **kw) == Status.ERR_INVALID_ARG
    assert err(opt.token_logprobs, x, targets, logp, logit_scale=-1.0) == Status.ERR_INVALID_ARG
    bf = x.bfloat16()
    wide = torch.zeros(T, V + 6, device="cuda")          # over the logits, but with another pitch
    same = wide.as_strided((T, V), (V, 1))
    assert err(opt.policy_loss, wide[:, :V], targets, old, adv, weights, same, stats) == Status.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        opt.policy_loss(x, targets, old, adv, weights, d[:, :-1], stats)
    with pytest.raises(ValueError):
        opt.policy_loss(x, targets[:-1], old, adv, weights, d, stats)
    with pytest.raises(ValueError):
        opt.policy_loss(x.t(), targets, old, adv, weights, d, stats)
    with pytest.raises(ValueError):
        opt.policy_loss(x, targets, old, adv, weights, d, stats[:3])
    with pytest.raises(TypeError):
        opt.policy_loss(x.half(), targets, old, adv, weights, d, stats)
    with pytest.raises(TypeError):
        opt.policy_loss(x, targets.int(), old, adv, weights, d, stats)
    with pytest.raises(TypeError):
        opt.policy_loss(x, targets, old.bfloat16(), adv, weights, d, stats)
    with pytest.raises(TypeError):
        opt.token_logprobs(bf.cpu(), targets, logp)
    assert opt.launch_count == 0 and not bool(d.any())
    empty = torch.empty(0, V, device="cuda")
    none = torch.empty(0, device="cuda")
    stats.fill_(5)
    opt.policy_loss(empty, none.long(), none, none, none, empty, stats)
    assert stats.tolist() == [0.0] * 4                                  # no rows: a sum of nothing
    opt.token_logprobs(empty, none.long(), none)
