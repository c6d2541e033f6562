"""Distillation rows whose teacher has no probability left, though their indices are valid: logits of -inf all over, or so far
below a given log-sum-exp that every probability is 0 in fp32.  Nothing is learned from such a row, whatever the student's
logits: its loss and gradient are 0, and where the student's row is not finite it adds 0 to all four sums."""
import math

import pytest
import torch

import paper_2305_19982_b200 as adama
from test_gpu_distill import FORMS, _case, _matrix, _outside_untouched

pytestmark = pytest.mark.gpu


def _spoiled(x, ids):
    """x with rows 0 to 3 not finite: all -inf; NaN at an entry; NaN elsewhere; +inf at an entry."""
    x = x.clone()
    x[0] = -math.inf
    x[1, ids[1, 3]] = math.nan
    x[2] = math.nan
    x[3 % x.shape[0], ids[3 % x.shape[0], 0]] = math.inf
    return x


@pytest.mark.parametrize("dtype,out", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T,V", FORMS)
@pytest.mark.parametrize("with_lse", [False, True])
def test_a_row_without_mass_is_neutral_whatever_the_student(T, V, dtype, out, with_lse):
    opt = adama.AdamA()
    K = 40
    _, x, t, ids, w = _case(T, V, K, dtype, torch.float32, V + 1, pitch=3, masked=0.0)
    x, dead = _spoiled(x, ids), list(range(4 if T > 4 else T - 1))
    if T < 4:                                            # three rows: one of them stays alive
        x[2] = x[2].nan_to_num(0.0)
    lse = None
    if with_lse:
        lse = torch.logsumexp(t, 1)
        lse[dead] = 1e4                                  # exp(t - 1e4) is 0 in fp32
        t[dead[0]] = -math.inf
    else:
        t[dead] = -math.inf
    buf, d = _matrix(T, V, out, 5, 1)
    stats, loss = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, teacher_lse=lse, loss=loss)
    # the same rows masked: not read at all
    w0 = w.clone()
    w0[dead] = 0.0
    _, d0 = _matrix(T, V, out, 5, 1)
    stats0, loss0 = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w0, d0, stats0, teacher_lse=lse, loss=loss0)
    assert bool(torch.isfinite(stats0).all()) and bool(torch.isfinite(d0).all())
    assert torch.equal(d, d0) and torch.equal(loss, loss0)
    assert float(d[dead].abs().max()) == 0 and float(loss[dead].abs().max()) == 0
    assert torch.equal(stats, stats0)
    _outside_untouched(buf, d)
    opt.distill_loss(x, t, ids, w, None, stats, teacher_lse=lse)          # the loss alone
    assert torch.equal(stats, stats0)
    if dtype == out:                                                      # the gradient replaces the logits
        opt.distill_loss(x, t, ids, w, x, stats, teacher_lse=lse)
        assert torch.equal(stats, stats0) and float(x[dead].abs().max()) == 0 and bool(torch.isfinite(x).all())
    opt.sync_status()


@pytest.mark.parametrize("T,V", FORMS)
def test_mass_on_one_entry_keeps_what_is_not_finite_visible(T, V):
    """One entry with probability: the row's NaN shows in its loss, its gradient and the sums, as for any other row."""
    opt = adama.AdamA()
    _, x, t, ids, w = _case(T, V, 40, torch.float32, torch.float32, V + 2, masked=0.0)
    x = _spoiled(x, ids)
    t[:2] = -math.inf
    t[:2, 5] = 0.0
    d, stats, loss = torch.empty(T, V, device="cuda"), torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats, loss=loss)
    assert bool(torch.isnan(loss[:2]).all()) and bool(torch.isnan(d[1]).all()) and bool(torch.isnan(stats[[0, 1, 2]]).all())
    opt.sync_status()


def test_a_finite_student_still_shows_what_it_holds_of_the_entries():
    """The third sum is the student's mass on the entries, with or without the teacher's."""
    opt = adama.AdamA()
    T, V, K = 6, 900, 10
    _, x, t, ids, w = _case(T, V, K, torch.float32, torch.float32, 5, masked=0.0)
    t[:] = -math.inf
    stats, d = torch.empty(4, device="cuda"), torch.empty(T, V, device="cuda")
    opt.distill_loss(x, t, ids, w, d, stats)
    held = float((w.double() * torch.softmax(x.double(), 1).gather(1, ids).sum(1)).sum())
    assert abs(float(stats[2]) - held) <= 4e-5 * held
    assert not bool(d.any()) and not bool(stats[[0, 1, 3]].any())
