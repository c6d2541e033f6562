"""The sign of a first moment held in 8 bits."""
import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import State8

pytestmark = pytest.mark.gpu
SIZES = [1, 3, 255, 256, 257, 4096, 50_021]


def _signs(codes):
    """-1, 0, 1 per e4m3 code: bit 7 is the sign, a code without it of 0 is zero."""
    c = codes.view(torch.uint8).cpu().numpy().astype(int)
    return np.where(c & 127, np.where(c & 128, -1, 1), 0)


@pytest.mark.parametrize("n", SIZES)
@pytest.mark.parametrize("offset", [0, 1])
def test_packed_moments_keep_their_signs(n, offset):
    """Every code that is not zero has its value's sign, and unpack gives it back."""
    opt = adama.AdamA()
    buf = torch.zeros(n + 4, device="cuda")
    m = buf[offset:offset + n]
    m.copy_(wl.normal((n,), 1e-3, torch.float32, n))
    s = State8.zeros(n)
    opt.state8_pack_multi([m], [torch.ones(n, device="cuda")], [s])
    got, want = _signs(s.m_codes), np.sign(m.cpu().numpy()).astype(int)
    assert np.array_equal(got, np.where(got != 0, want, 0)) and np.count_nonzero(got) >= 0.9 * n
    um, uv = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    opt.state8_unpack_multi([s], [um], [uv])
    assert np.array_equal(np.sign(um.cpu().numpy()).astype(int), got)


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", SIZES + [3_000_001])           # the last one is streamed
def test_updated_moments_have_the_signs_of_the_formula(n, gdtype):
    """Three steps with gradients of either sign: m in 64 bits, from the state that the call was given.  Where
    |m| is beyond the smallest code's reach (a half of 2^-9 of the scale, and the rounding of m itself,
    2^-22 of its terms) its code has its sign, and no code has the other one."""
    opt = adama.AdamA()
    w, s = torch.zeros(n, device="cuda"), State8.zeros(n)
    um, uv = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    for step in range(3):
        g = wl.normal((n,), 1e-3, torch.float32, 10 * n + step).to(gdtype).cuda()
        opt.state8_unpack_multi([s], [um], [uv])
        a = float(np.float32(1 - 0.9))
        m = um.double().cpu().numpy() + a * g.double().cpu().numpy()
        terms = np.abs(um.double().cpu().numpy()) + a * np.abs(g.double().cpu().numpy())
        opt.begin_minibatch(1)
        opt.fold_apply8_multi([w], [g], [s], wl.LR)
        got = _signs(s.m_codes)
        blocks = np.zeros(-(-n // 256) * 256)
        blocks[:n] = np.abs(m)
        scale = np.repeat(blocks.reshape(-1, 256).max(1) / 448.0, 256)[:n]
        sure = np.abs(m) > 2.0 ** -10 * scale * (1 + 1e-5) + 2.0 ** -22 * terms
        assert sure.mean() >= 0.9 and np.array_equal(got[sure], np.sign(m[sure]).astype(int))
        unsure = ~sure & (np.abs(m) > 2.0 ** -22 * terms)
        assert not np.any(got[unsure] * np.sign(m[unsure]) < 0)
    opt.sync_status()
