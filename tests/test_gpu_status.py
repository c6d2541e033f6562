"""What the device reports to the host: an expired wait and a target outside the vocabulary do not hide
each other."""
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu


def _bad_target(opt):
    x = wl.normal((5, 50), 1.0, torch.float32, 1).cuda()
    opt.token_logprobs(x, torch.tensor([1, 2, 3, 50, 4]).cuda(), torch.empty(5, device="cuda"))


def _expired_wait(opt):
    """The fused kernel with waits of 1 ms, one of which runs out; it returns by itself."""
    opt.begin_minibatch(1)
    X = wl.small_integers((256, 512), 2, torch.bfloat16, 1).cuda()
    dY = wl.small_integers((256, 768), 2, torch.bfloat16, 2).cuda()
    m, v = torch.zeros(512, 768, device="cuda"), torch.zeros(512, 768, device="cuda")
    opt.debug_wgrad_expire_wait(X, dY, m, v, wait_limit_ns=1_000_000)


@pytest.mark.parametrize("order", [(_bad_target, _expired_wait), (_expired_wait, _bad_target)])
def test_a_bad_target_and_an_expired_wait_are_both_reported(order):
    opt = adama.AdamA()
    for call in order:
        call(opt)
    with pytest.raises(adama.AdamAError) as e:
        opt.sync_status()                                    # the incomplete m and v come first
    assert e.value.status == Status.ERR_TIMEOUT and "wait" in str(e.value)
    with pytest.raises(adama.AdamAError) as e:
        opt.sync_status()
    assert e.value.status == Status.ERR_INVALID_ARG and "row 3" in str(e.value)
    opt.sync_status()                                        # each is cleared by its report


def test_the_first_bad_row_of_a_call_that_follows_a_report_is_named():
    opt = adama.AdamA()
    for _ in range(2):
        _bad_target(opt)
        with pytest.raises(adama.AdamAError) as e:
            opt.sync_status()
        assert "row 3" in str(e.value)
    opt.sync_status()
