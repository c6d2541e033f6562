"""Distillation from a teacher's top logits (adama_distill_loss) against the definition in 64 bits.

Tolerances.  LOGP = 1e-5 bounds the student's log-probabilities for |z - lse| <= 60 and rows of at most 2^19
elements (a thread adds at most 2^19/512 terms one after the other, whose roundings' random walk stays under 2e-6; the
exponentials' arguments carry 60*2^-24, the exponentials 2^-22), and with fewer terms the teacher's.  So p and q are off
by 1e-5 + 2^-22 relative, a product of P and q by PQ = 3e-5.  A row's divergence: sum p*(2*LOGP) + 1.1e-5*sum p*|log p - log q|.  The
gradient: unit*(PQ*P*q + 2e-5*own), own the sum of p over the entries of an index, plus half a last place."""
import math

import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu
LOGP, PQ = 1e-5, 3e-5
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
SENTINEL = 777.0


def _matrix(rows, cols, dtype, pitch=0, offset=0, values=None):
    ld = cols + pitch
    buf = torch.full((offset + rows * ld + 64,), SENTINEL, dtype=dtype, device="cuda")
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    if values is not None:
        view.copy_(values)
    return buf, view


def _outside_untouched(buf, view):
    mask = torch.ones_like(buf, dtype=torch.bool)
    at = view.storage_offset() - buf.storage_offset()
    mask[at:at + view.shape[0] * view.stride(0)].view(view.shape[0], view.stride(0))[:, :view.shape[1]] = False
    assert bool((buf[mask] == SENTINEL).all())


def _case(T, V, K, dtype, teacher, seed, pitch=0, offset=0, masked=0.25):
    g = torch.Generator().manual_seed(seed)
    buf, x = _matrix(T, V, dtype, pitch, offset, wl.normal((T, V), 2.0, torch.float32, seed))
    _, t = _matrix(T, K, teacher, 5, 1, wl.normal((T, K), 2.0, torch.float32, seed + 1))
    ids = torch.stack([torch.randperm(V, generator=g)[:K] if V <= 20_000 else torch.randint(0, V, (K,), generator=g) for _ in range(T)])
    wide = torch.full((T, K + 3), -9, dtype=torch.int64, device="cuda")
    wide[:, :K] = ids
    w = torch.rand(T, generator=g) + 0.5
    w[torch.rand(T, generator=g) < masked] = 0.0
    return buf, x, t, wide[:, :K], w.cuda()


def _reference(x, t, ids, w, lse, scale):
    """In float64: per-row kl, cross entropy, mass held, P; the gradient and the parts that its tolerance needs."""
    x, t, ids, w = x.double().cpu(), t.double().cpu() * scale, ids.cpu(), w.double().cpu()
    logq = torch.log_softmax(x * scale, 1)
    t = torch.where(ids >= 0, t, -math.inf)
    some = (t > -math.inf).any(1)
    logp = t - (torch.where(some, torch.logsumexp(t, 1), 0.0) if lse is None else lse.double().cpu())[:, None]
    p = torch.exp(logp)
    at = logq.gather(1, ids.clamp(min=0))
    zero = torch.zeros_like(p)
    kl = torch.where(p > 0, p * (logp - at), zero).sum(1)
    far = torch.where(p > 0, p * (logp - at).abs(), zero).sum(1)
    cross = -torch.where(p > 0, p * at, zero).sum(1)
    held, P = torch.where(ids >= 0, at.exp(), zero).sum(1), p.sum(1)
    q = torch.exp(logq)
    own = torch.zeros_like(q).scatter_add_(1, ids.clamp(min=0), p)
    unit = (w * scale)[:, None]
    grad = unit * (P[:, None] * q - own)
    bound = unit.abs() * (PQ * P[:, None] * q + 2e-5 * own)
    live = w != 0
    clean = lambda r: torch.where(live, r, 0.0)  # noqa: E731
    return dict(kl=clean(kl), far=clean(far), cross=clean(cross), held=clean(held), P=clean(P), w=w,
                grad=torch.where(live[:, None], grad, 0.0), bound=torch.where(live[:, None], bound, 0.0))


def _check(r, d, stats, loss):
    kl_tol = 2 * LOGP * r["P"] + 1.1e-5 * r["far"]
    assert bool(((loss.cpu().double() - r["kl"]).abs() <= kl_tol + 2.0 ** -23 * r["kl"].abs()).all())
    w = r["w"].abs()
    tols = (kl_tol + 2.0 ** -23 * r["kl"].abs(), 2e-5 * (r["P"] + r["cross"].abs()), PQ * r["held"], PQ * r["P"])
    for got, key, tol in zip(stats.tolist(), ("kl", "cross", "held", "P"), tols):
        want = float((r["w"] * r[key]).sum())
        assert abs(got - want) <= float((w * tol).sum()) + 2.0 ** -23 * abs(want), key
    if d is not None:
        g = d.cpu().double()
        assert bool(((g - r["grad"]).abs() <= r["bound"] + HALF_ULP[d.dtype] * (r["grad"].abs() + r["bound"])).all())


# rows in registers; rings of 64, 128, 256, 512 and 640 threads; clusters, one row and several rows to each; rows read twice
SHAPES = [(1, 1, 1), (3, 7, 2), (5, 100, 33), (4, 1000, 64), (300, 513, 20), (700, 2040, 128), (900, 4099, 31), (2000, 6001, 100), (1, 9001, 1), (700, 9001, 100),
          (400, 20_011, 65), (200, 32_768, 10), (200, 50_257, 50), (33, 131_072, 20), (300, 131_072, 64), (3, 480_001, 100)]


@pytest.mark.parametrize("dtype,out,teacher", [(torch.float32, torch.float32, torch.float32), (torch.float32, torch.bfloat16, torch.bfloat16),
                                               (torch.bfloat16, torch.bfloat16, torch.float32), (torch.bfloat16, torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,V,K", SHAPES)
@pytest.mark.parametrize("pitch,offset,scale,with_lse", [(0, 0, 1.0, False), (5, 3, 0.5, True)])
def test_loss_and_gradient(T, V, K, dtype, out, teacher, pitch, offset, scale, with_lse):
    opt = adama.AdamA()
    _, x, t, ids, w = _case(T, V, K, dtype, teacher, T + V, pitch, offset)
    lse = None
    if with_lse:
        lse = (torch.logsumexp(t.float() * scale, 1) + 0.125 * torch.rand(T, generator=torch.Generator().manual_seed(1)).cuda())
    buf, d = _matrix(T, V, out, pitch + 2, offset)
    stats, loss = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, teacher_lse=lse, loss=loss, logit_scale=scale)
    r = _reference(x, t, ids, w, lse, scale)
    _check(r, d, stats, loss)
    _outside_untouched(buf, d)
    assert float(d[w == 0].abs().max()) == 0 if bool((w == 0).any()) else True
    first = d.clone(), stats.clone()
    opt.distill_loss(x, t, ids, w, d, stats, teacher_lse=lse, logit_scale=scale)
    assert torch.equal(d, first[0]) and torch.equal(stats, first[1])       # bit for bit
    opt.distill_loss(x, t, ids, w, None, stats, teacher_lse=lse, loss=loss, logit_scale=scale)
    assert torch.equal(stats, first[1])                                    # the loss alone
    if dtype == out and pitch == 0:                                        # the gradient replaces the logits
        opt.distill_loss(x, t, ids, w, x, stats, teacher_lse=lse, logit_scale=scale)
        assert torch.equal(stats, first[1])
        err = (x.cpu().double() - r["grad"]).abs()
        assert bool((err <= r["bound"] + HALF_ULP[out] * (r["grad"].abs() + r["bound"])).all())
    opt.sync_status()


FORMS = [(40, 300), (40, 2040), (40, 5000), (200, 5000), (40, 20_000), (300, 60_001), (3, 480_001)]


@pytest.mark.parametrize("T,V", FORMS)
def test_entries_left_out_and_entries_twice(T, V):
    """Negative indices, teacher's logits of -inf, rows of nothing else, the same index two to many times."""
    opt = adama.AdamA()
    K = 100
    _, x, t, ids, w = _case(T, V, K, torch.float32, torch.float32, V, masked=0.0)
    ids[:, 3] = -1
    ids[0, 40:] = -5                                     # 39 left
    ids[1] = -1                                          # none
    t[2] = -math.inf                                     # none either
    t[0, 7] = -math.inf
    if T > 3:
        ids[3] = 17                                      # one index, a hundred times
        t[4 % T, 1:] = -math.inf                         # one entry: probability 1
        ids[5, 99], ids[5, 64], ids[5, 33] = ids[5, 0], ids[5, 0], ids[5, 32]
        ids[6, 1:3] = ids[6, 0]
        ids[7, 50] = V - 1
        ids[8, 50], ids[8, 51] = 0, 0
    d, stats, loss = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    r = _reference(x, t, ids, w, None, 1.0)
    _check(r, d, stats, loss)
    for row in (1, 2):
        assert float(loss[row]) == 0 and float(d[row].abs().max()) == 0
    opt.sync_status()


@pytest.mark.parametrize("T,V", FORMS)
def test_rows_that_are_not_finite(T, V):
    opt = adama.AdamA()
    _, x, t, ids, w = _case(T, V, 20, torch.float32, torch.float32, V, masked=0.0)
    clean, stats, loss = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, clean, stats)
    x[0, :] = -math.inf                                  # nothing left of the student
    x[1, :] = torch.finfo(torch.float32).min             # the type's lowest value all over: even
    x[2, V // 2] = math.nan
    ids[1] = torch.arange(20, device="cuda")
    d = torch.empty(T, V, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    assert math.isnan(float(loss[0])) and math.isnan(float(loss[2])) and torch.isnan(d[2]).all()
    p = torch.softmax(t[1].double(), 0)
    assert abs(float(loss[1]) - float((p * (p.log() + math.log(V))).sum())) <= 3e-5
    assert abs(float(d[1, V - 1]) - float(w[1]) / V) <= 4e-5 * float(w[1]) / V
    assert torch.equal(d[3:], clean[3:])
    x[:, :] = 0.0
    x[0, ids[0, 4]] = -math.inf                          # the student has none of what the teacher has
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    assert float(loss[0]) == math.inf and torch.isfinite(d).all()
    x[0, :] = -math.inf                                  # a row that has no entry either
    ids[0] = -1
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    assert float(loss[0]) == 0 and float(d[0].abs().max()) == 0 and math.isfinite(float(stats[0]))
    w[0] = 0.0
    x[0, :] = math.nan                                   # a row without weight is not read
    opt.distill_loss(x, t, ids, w, d, stats)
    assert float(d[0].abs().max()) == 0 and math.isfinite(float(stats[0]))


@pytest.mark.parametrize("T,V", FORMS)
def test_an_index_outside_the_vocabulary_is_reported(T, V):
    opt = adama.AdamA()
    _, x, t, ids, w = _case(T, V, 40, torch.bfloat16, torch.float32, V, masked=0.0)
    ids[1, 35] = V
    ids[2, 0] = 1 << 40
    d, stats, loss = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    assert torch.isnan(d[1:3]).all() and torch.isnan(loss[1:3]).all() and math.isnan(float(stats[0]))
    assert torch.isfinite(d[0]).all() and math.isfinite(float(loss[0])) and torch.isfinite(d[3:]).all()
    with pytest.raises(adama.AdamAError) as e:
        opt.sync_status()
    assert e.value.status == Status.ERR_INVALID_ARG
    opt.sync_status()


def test_a_common_offset_costs_no_precision():
    opt = adama.AdamA()
    T, V, K = 4, 5000, 20
    x = (torch.randint(-200, 200, (T, V), generator=torch.Generator().manual_seed(1)) / 64.0).cuda()
    t = (torch.randint(-200, 200, (T, K), generator=torch.Generator().manual_seed(2)) / 64.0).cuda()
    ids = torch.arange(T * K, device="cuda").view(T, K)
    out = []
    for shift in (0.0, 4096.0):
        d, stats = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")
        opt.distill_loss(x + shift, t + shift, ids, torch.ones(T, device="cuda"), d, stats)
        out.append((d, stats))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_gradient_against_differences():
    opt = adama.AdamA()
    T, V, K = 2, 9, 4
    _, x, t, ids, w = _case(T, V, K, torch.float32, torch.float32, 3, masked=0.0)
    ids[1, 2] = ids[1, 0]
    lse = torch.logsumexp(t * 0.5, 1) + 0.3
    d, stats = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, teacher_lse=lse, logit_scale=0.5)
    base = x.double().cpu()
    for at in np.ndindex(T, V):
        plus, minus = base.clone(), base.clone()
        plus[at] += 1e-5
        minus[at] -= 1e-5
        loss = [float((r["w"] * r["kl"]).sum()) for r in (_reference(y, t, ids, w, lse, 0.5) for y in (plus, minus))]
        assert abs(float(d[at]) - (loss[0] - loss[1]) / 2e-5) <= 1e-4


def test_captured_and_played_again():
    opt = adama.AdamA()
    _, x, t, ids, w = _case(300, 3000, 40, torch.bfloat16, torch.float32, 3)
    d, stats = torch.empty(300, 3000, dtype=torch.bfloat16, device="cuda"), torch.empty(4, device="cuda")
    want_d, want = torch.empty_like(d), torch.empty_like(stats)
    opt.distill_loss(x, t, ids, w, want_d, want)
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g):
            opt.distill_loss(x, t, ids, w, d, stats)
    for g in (graphs[1], graphs[0], graphs[1]):
        d.zero_()
        stats.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(d, want_d) and torch.equal(stats, want)


def test_no_rows():
    opt = adama.AdamA()
    stats = torch.full((4,), SENTINEL, device="cuda")
    x, t = torch.empty(0, 50, device="cuda"), torch.empty(0, 4, device="cuda")
    opt.distill_loss(x, t, t.long(), torch.empty(0, device="cuda"), torch.empty_like(x), stats)
    assert float(stats.abs().max()) == 0
    opt.sync_status()


def test_refusals():
    opt = adama.AdamA()
    T, V, K = 3, 50, 5
    _, x, t, ids, w = _case(T, V, K, torch.float32, torch.float32, 1)
    d, stats = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda")

    def refused(kind, *args, **kw):
        with pytest.raises(kind) as e:
            opt.distill_loss(*args, **kw)
        return e.value

    refused(ValueError, x, t[:2], ids, w, d, stats)
    refused(ValueError, x, t, ids[:, :4], w, d, stats)
    refused(ValueError, x, t, ids, w[:2], d, stats)
    refused(ValueError, x, t, ids, w, d[:, :49], stats)
    refused(ValueError, x, t, ids, w, d, stats[:3])
    refused(ValueError, x, t, ids, w, d, stats, teacher_lse=w[:2])
    refused(ValueError, x, t, ids.t().contiguous().t(), w, d, stats)
    refused(TypeError, x, t, ids.int(), w, d, stats)
    refused(TypeError, x, t.half(), ids, w, d, stats)
    refused(TypeError, x, t, ids.cpu(), w, d, stats)
    many = torch.zeros(T, 129, device="cuda")
    assert refused(adama.AdamAError, x, many, many.long(), w, d, stats).status == Status.ERR_UNSUPPORTED
    assert refused(adama.AdamAError, x, many[:, :0], many[:, :0].long(), w, d, stats).status == Status.ERR_INVALID_ARG
    for scale in (0.0, -1.0, math.nan, 1e39):
        assert refused(adama.AdamAError, x, t, ids, w, d, stats, logit_scale=scale).status == Status.ERR_INVALID_ARG
    opt.sync_status()


@pytest.mark.parametrize("T,V,dtype", [(2000, 6000, torch.float32), (2000, 12_000, torch.bfloat16), (500, 60_000, torch.bfloat16)])
def test_results_repeat_to_the_bit(T, V, dtype):
    """Many runs, since a stage of the ring that were filled anew while it is still read would show in few of them."""
    opt = adama.AdamA()
    _, x, t, ids, w = _case(T, V, 100, dtype, torch.float32, T + V)
    _, d = _matrix(T, V, torch.bfloat16, 2)
    stats, loss = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    first = None
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(400):
        opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
        if first is None:
            first = [r.clone() for r in (d, stats, loss)]
        differ += sum((a != b).any() for a, b in zip((d, stats, loss), first))
    assert int(differ) == 0
    opt.sync_status()
