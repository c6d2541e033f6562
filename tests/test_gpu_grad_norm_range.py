"""The gradient norm over the range that its fp32 squares allow: 64 of them in one sum stay finite up to
entries of 2.3e18, and are normal numbers from entries of 1.1e-19 on."""
import math

import pytest
import torch

import paper_2305_19982_b200 as adama

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 70_001])
@pytest.mark.parametrize("size", [2.2e18, 1e18, 1e-18, 1.2e-19])
def test_the_norm_holds_within_its_range(n, size, gdtype):
    opt = adama.AdamA()
    g = torch.full((n,), size, device="cuda").to(gdtype)
    g[1::2] *= -1
    out = torch.empty(4, device="cuda")
    opt.grad_norm_multi([g], 1.0, out)
    want = math.sqrt(float(g.double().square().sum()))
    assert abs(float(out[0]) - want) <= 6e-7 * want
    assert abs(float(out[1]) - min(1.0, 1.0 / want)) <= 7e-7 * min(1.0, 1.0 / want)


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
def test_beyond_it_the_step_is_skipped_or_the_entries_vanish(gdtype):
    """One entry of 1.9e19 has a square beyond fp32: the factor is NaN.  Entries of 1e-23 add nothing."""
    opt = adama.AdamA()
    out = torch.empty(4, device="cuda")
    g = torch.full((5000,), 1e-23, device="cuda").to(gdtype)
    opt.grad_norm_multi([g], 1.0, out)
    assert out[:2].tolist() == [0.0, 1.0]
    g[77] = 1.9e19
    opt.grad_norm_multi([g], 1.0, out)
    assert not math.isfinite(float(out[0])) and math.isnan(float(out[1]))
