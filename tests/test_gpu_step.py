"""The one-pass update of many tensors (adama_fold_apply_multi, adama_fold_apply8_multi), the 8-bit
state format and the gradient norm with its clip factor."""
import math

import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from oracle import AdamAOracle
from paper_2305_19982_b200 import State8, State8List, Status
from parity import Guarded, f64, rel_l2

pytestmark = pytest.mark.gpu
TOL = 1e-6        # fp32 state, a handful of roundings of 2^-24 per mini-batch (as for fold and apply)
F = np.float32


def _views(sizes, offset_by, dtype=torch.float32):
    """One tensor per size with mixed alignment (0..3 elements past a 16-byte boundary)."""
    return [torch.zeros(n + 8, dtype=dtype, device="cuda")[(i * offset_by) % 4:(i * offset_by) % 4 + n]
            for i, n in enumerate(sizes)]


# ---- 32-bit states -------------------------------------------------------------------------------

SIZES = [1, 2, 3, 4, 5, 255, 4095, 4096, 4097, 0, 8192, 12_289, 100_003]


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("steps_w,steps_g", [(0, 0), (1, 1), (1, 0), (2, 3), (0, 1)])
def test_fold_apply_equals_fold_then_apply_and_oracle(gdtype, steps_w, steps_g):
    """Bit for bit what adama_fold_multi and adama_apply_multi give, for every alignment: w, m, v
    aligned alike or not, the gradient reaching its boundary with them or not."""
    N = 3
    w0 = [wl.normal((n,), 0.02, torch.float32, 100 + i) for i, n in enumerate(SIZES)]
    one = [_views(SIZES, s) for s in (steps_w, steps_w, steps_w)]
    two = [[x.clone() for x in xs] for xs in one]
    for xs in (one[0], two[0]):
        for x, y in zip(xs, w0):
            x.copy_(y)
    copies = _views(SIZES, steps_g, torch.bfloat16)
    orcs = [AdamAOracle(f64(x)) for x in w0]
    a, b = adama.AdamA(), adama.AdamA()
    for opt in (a, b):
        opt.set_weight_decay(0.0)
    for step in range(2):
        a.begin_minibatch(N)
        b.begin_minibatch(N)
        for o in orcs:
            o.begin_minibatch(N)
        for i in range(N):
            host = [wl.normal((n,), 1e-2, gdtype, 7000 + 1000 * step + 200 * i + k) for k, n in enumerate(SIZES)]
            grads = _views(SIZES, steps_g, gdtype)
            for g, h in zip(grads, host):
                g.copy_(h)
            b.fold_multi(grads, two[1], two[2])
            if i < N - 1:
                a.fold_multi(grads, one[1], one[2])
            else:
                a.fold_apply_multi(one[0], grads, one[1], one[2], wl.LR, w_bf16=copies)
            for o, h in zip(orcs, host):
                if h.numel():
                    o.fold(f64(h))
        b.apply_multi(two[0], two[1], two[2], wl.LR)
        for o, n in zip(orcs, SIZES):
            if n:
                o.update(wl.LR)
        for x, y in zip(one[0] + one[1] + one[2], two[0] + two[1] + two[2]):
            assert torch.equal(x, y)
        for x, y in zip(copies, two[0]):
            assert torch.equal(x, y.bfloat16())
        for k in (6, 8, 12):
            assert rel_l2(f64(one[0][k]), orcs[k].theta) <= TOL
            assert rel_l2(f64(one[2][k]), wl.BETA2 * orcs[k].v) <= TOL
    a.close()
    b.close()


def test_fold_apply_more_tensors_than_one_launch_holds():
    sizes = [(37 * i) % 300 for i in range(1100)]
    opt, ref = adama.AdamA(), adama.AdamA()
    ws, ms, vs, gs = ([wl.normal((n,), 0.02, torch.float32, k * 5000 + i).cuda() for i, n in enumerate(sizes)]
                      for k in range(4))
    vs = [v.abs() for v in vs]
    w2, m2, v2 = ([x.clone() for x in xs] for xs in (ws, ms, vs))
    for o in (opt, ref):
        o.set_step(7)
        o.begin_minibatch(1)
    opt.fold_apply_multi(ws, gs, ms, vs, wl.LR)
    assert opt.launch_count == 3                # 1100 tensors, at most 512 in a launch
    ref.fold_multi(gs, m2, v2)
    ref.apply_multi(w2, m2, v2, wl.LR)
    for x, y in zip(ws + ms + vs, w2 + m2 + v2):
        assert torch.equal(x, y)


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,g_offset", [(1, 3), (1, 1), (3, 3), (2, 6), (3, 7)])
@pytest.mark.parametrize("n", [1, 2, 4, 7, 4099, 70_001])
def test_fold_apply_writes_nothing_outside_its_tensors(n, offset, g_offset, gdtype):
    """Among them tensors that end before the first boundary that their vector accesses wait for."""
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    bufs = [Guarded(n, offset=offset).zero() for _ in range(3)]
    copy = Guarded(n, dtype=torch.bfloat16, offset=g_offset).zero()
    g = Guarded(n, dtype=gdtype, offset=g_offset).fill(wl.normal((n,), 1e-2, gdtype, 5).cuda())
    opt.fold_apply_multi([bufs[0].view], [g.view], [bufs[1].view], [bufs[2].view], wl.LR, w_bf16=[copy.view])
    for b in bufs + [copy, g]:
        b.check()
    assert bool((bufs[0].view != 0).all())


LONG = [2_500_001, 1, 6, 2048, 700_003, 4095, 1_048_576, 3]     # long enough to be streamed through shared memory


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset,g_offset", [(0, 0), (1, 1), (3, 3), (2, 6), (1, 5), (0, 2), (1, 0), (0, 4), (3, 1)])
def test_long_lists_equal_fold_then_apply(gdtype, offset, g_offset):
    """Heads before the first boundary, ragged ends, gradients that reach their boundary with the
    weights or not, chunks of one tensor beside those of the next; nothing outside is written."""
    bufs = [[Guarded(n, offset=offset) for n in LONG] for _ in range(3)]
    copies = [Guarded(n, dtype=torch.bfloat16, offset=offset) if i != 4 else None for i, n in enumerate(LONG)]
    grads = [Guarded(n, dtype=gdtype, offset=g_offset) for n in LONG]
    gen = torch.Generator(device="cuda").manual_seed(offset + 10 * g_offset)
    for k, bs in enumerate(bufs):
        for b in bs:
            b.view.copy_(torch.randn(b.n, generator=gen, device="cuda") * 0.02)
            if k == 2:
                b.view.square_()
    for g in grads:
        g.view.copy_((torch.randn(g.n, generator=gen, device="cuda") * 1e-2).to(gdtype))
    for c in copies:
        if c is not None:
            c.zero()
    w2, m2, v2 = ([b.view.clone() for b in bs] for bs in bufs)
    a, b = adama.AdamA(), adama.AdamA()
    for opt in (a, b):
        opt.set_step(5)
        opt.begin_minibatch(1)
        opt.set_weight_decay(0.01)
    gs = [g.view for g in grads]
    a.fold_apply_multi(*([x.view for x in bs] for bs in bufs[:1]), gs, *([x.view for x in bs] for bs in bufs[1:]), wl.LR,
                       w_bf16=[c.view if c is not None else None for c in copies])
    assert a.launch_count == 1
    b.fold_multi(gs, m2, v2)
    b.apply_multi(w2, m2, v2, wl.LR)
    a.sync_status()
    for bs, want in zip(bufs, (w2, m2, v2)):
        for x, y in zip(bs, want):
            assert torch.equal(x.view, y)
            x.check()
    for c, y in zip(copies, w2):
        if c is not None:
            assert torch.equal(c.view, y.bfloat16())
            c.check()
    for g in grads:
        g.check()


def test_factor_multiplies_the_gradient_and_nan_skips_the_step():
    n = 10_001
    g = wl.normal((n,), 1e-2, torch.float32, 1).cuda()
    factor = torch.tensor([0.37], device="cuda")
    res = []
    for scaled in (False, True):
        opt = adama.AdamA()
        opt.set_weight_decay(0.01)
        w = wl.normal((n,), 0.02, torch.float32, 2).cuda()
        m, v = torch.zeros_like(w), torch.zeros_like(w)
        copy = torch.full((n,), 3.0, dtype=torch.bfloat16, device="cuda")
        opt.begin_minibatch(1)
        opt.fold_apply_multi([w], [g * factor if scaled else g], [m], [v], wl.LR, w_bf16=[copy],
                             grad_factor=None if scaled else factor)
        res.append((w, m, v, copy))
    assert all(torch.equal(x, y) for x, y in zip(*res))
    before = [t.clone() for t in (w, m, v, copy)]
    opt.begin_minibatch(1)
    opt.fold_apply_multi([w], [g], [m], [v], wl.LR, w_bf16=[copy], grad_factor=torch.full((1,), math.nan, device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(before, (w, m, v, copy)))
    s = State8.zeros(n)
    opt.fold_apply8_multi([w], [g], [s], wl.LR, w_bf16=[copy], grad_factor=torch.full((1,), math.nan, device="cuda"))
    assert torch.equal(before[0], w) and torch.equal(before[3], copy)
    assert not bool(s.m_scale.any()) and not bool(s.v_scale.any()) and not bool(s.v_codes.any())


# ---- 8-bit states ----------------------------------------------------------------------------------

def _v_values():
    c = np.arange(256)
    return np.where(c > 0, (1 + (c % 8) / 8) * 2.0 ** (c // 8 - 31), 0.0)


def _e4m3_values():
    """The 256 e4m3 codes' values, from the format's definition (bias 7, 0x7f and 0xff NaN)."""
    out = np.zeros(256)
    for c in range(256):
        s, e, f = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        out[c] = math.nan if c & 127 == 127 else s * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
    return out


def _decode(s: State8):
    """m, v of a state in float64, from the codes and scales as documented."""
    rep = lambda t: np.repeat(f64(t), 256)[:s.numel]  # noqa: E731
    mc, vc = s.m_codes.view(torch.uint8).cpu().numpy(), s.v_codes.cpu().numpy()
    return _e4m3_values()[mc] * rep(s.m_scale), _v_values()[vc] * rep(s.v_scale)


def _blocks(x):
    pad = np.zeros(-(-x.size // 256) * 256, dtype=x.dtype)
    pad[:x.size] = x
    return pad.reshape(-1, 256)


def _check_rounded(got, want, top_code, values, unsigned):
    """Every element is within half the distance between the code values around it (times 1 + 2e-6
    for the fp32 arithmetic before the rounding); nothing is above the block's largest."""
    want_b, got_b = _blocks(want), _blocks(got)
    scale = np.abs(want_b).max(1, keepdims=True) / top_code
    safe = np.where(scale > 0, scale, 1.0)
    y, z = np.abs(want_b / safe), np.abs(got_b / safe)
    values = np.unique(np.abs(values[np.isfinite(values)]))
    hi = np.clip(np.searchsorted(values, y), 1, len(values) - 1)
    half = (values[hi] - values[hi - 1]) / 2
    if unsigned:                                # not rounded to zero: the smallest code stands in
        half = np.where(y < values[1], values[1], half)
    assert np.all(np.abs(z - y) <= half * (1 + 1e-5) + 2e-6 * y)
    return y, z


@pytest.mark.parametrize("n", [1, 3, 255, 256, 257, 4096, 5000, 70_001])
@pytest.mark.parametrize("offset", [0, 1])
def test_pack_rounds_to_the_nearest_code_and_unpack_reads_it(n, offset):
    opt = adama.AdamA()
    spread = torch.exp(4 * wl.normal((n,), 1.0, torch.float32, 3))
    m = Guarded(n, offset=offset).fill((wl.normal((n,), 1e-3, torch.float32, 1) * spread).cuda())
    v = Guarded(n, offset=offset).fill((wl.normal((n,), 1e-3, torch.float32, 2) * spread).square().cuda())
    s = State8.zeros(n)
    opt.state8_pack_multi([m.view], [v.view], [s])
    dm, dv = _decode(s)
    _check_rounded(dm, f64(m.view), 448.0, _e4m3_values(), False)
    _check_rounded(dv, f64(v.view), 1.875, _v_values(), True)
    assert np.all((dv > 0) == (f64(v.view) > 0))
    um, uv = Guarded(n, offset=offset), Guarded(n, offset=offset)
    opt.state8_unpack_multi([s], [um.view], [uv.view])
    for b in (m, v, um, uv):
        b.check()
    # code times scale, one fp32 rounding
    assert np.array_equal(f64(um.view), dm.astype(F).astype(float)) and np.array_equal(f64(uv.view), dv.astype(F).astype(float))
    # the values of an unpack are code values again: packing them changes the scale's last bit at most
    s2 = State8.zeros(n)
    opt.state8_pack_multi([um.view], [uv.view], [s2])
    assert torch.equal(s.v_codes, s2.v_codes)
    assert torch.equal(s.m_codes.view(torch.uint8) & 127, s2.m_codes.view(torch.uint8) & 127)
    assert torch.allclose(s.m_scale, s2.m_scale, rtol=2.5e-7, atol=0) and torch.allclose(s.v_scale, s2.v_scale, rtol=2.5e-7, atol=0)


def test_pack_ties_go_to_the_even_code_and_the_range_ends_hold():
    opt = adama.AdamA()
    m = torch.zeros(256)
    m[:9] = torch.tensor([448.0, 1.0625, 1.1875, -1.0625, 2.0 ** -10, 1.5 * 2.0 ** -9, 2.5 * 2.0 ** -9, 2.0 ** -11, -448.0])
    v = torch.zeros(256)
    v[:7] = torch.tensor([1.875, 1.0625, 1.1875, 2.0 ** -31, 2.0 ** -40, 1e-37, 0.0])
    s = State8.zeros(256)
    opt.state8_pack_multi([m.cuda()], [v.cuda()], [s])
    dm, dv = _decode(s)
    # 448 and 1.875 at the top make the scales 448*(1/448) and 1.875*(1/1.875): 1 to the last bit
    assert np.allclose(dm[:9], [448, 1.0, 1.25, -1.0, 0, 2 * 2.0 ** -9, 2 * 2.0 ** -9, 0, -448], rtol=2e-7, atol=0)
    low = float(_v_values()[1])
    assert np.allclose(dv[:7], [1.875, 1.0, 1.25, low, low, low, 0], rtol=2e-7, atol=0)
    assert s.v_codes[3:7].tolist() == [1, 1, 1, 0]


def _emulate_step8(w, g, s, t, lr, factor, wd):
    """The call's arithmetic in numpy fp32, operation by operation; returns w in float64 (its update
    uses approximate roots) and the codes and scales bit for bit."""
    n = w.size
    a, b = F(1 - 0.9), F(1 - 0.999)
    rep = lambda x: np.repeat(x.cpu().numpy(), 256)[:n]  # noqa: E731
    m = (_e4m3_values().astype(F)[s.m_codes.view(torch.uint8).cpu().numpy()] * rep(s.m_scale)).astype(F)
    v = (_v_values().astype(F)[s.v_codes.cpu().numpy()] * rep(s.v_scale)).astype(F)
    g = (g.astype(F) * F(factor)).astype(F)
    m = (m + (g * a).astype(F)).astype(F)
    v = (v + ((g * b).astype(F) * g).astype(F)).astype(F)
    step, ibc2 = F(lr / (1 - 0.9 ** t)), F(1 / (1 - 0.999 ** t))
    w64 = w.astype(float) * float(F(1 - lr * wd)) - float(step) * m.astype(float) / (
        np.sqrt(v.astype(float) * float(ibc2)) + float(F(1e-8)))
    mb, vb = _blocks(m), _blocks(v)
    mt, vt = np.abs(mb).max(1, keepdims=True), vb.max(1, keepdims=True)
    big = np.finfo(F).max
    with np.errstate(divide="ignore", over="ignore"):
        mi = np.minimum(((F(1) / mt).astype(F) * F(448)).astype(F), big)
        vi = np.minimum(((F(1) / vt).astype(F) * F(1.875)).astype(F), big)
    codes_m = torch.from_numpy((mb * mi).astype(F)).to(torch.float8_e4m3fn).view(torch.uint8).numpy().reshape(-1)[:n]
    bits = (vb * vi).astype(F).view(np.int32).astype(np.int64)
    codes_v = np.clip(((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - 768, 1, 255)
    codes_v = np.where(vb > 0, codes_v, 0).reshape(-1)[:n]
    sm = ((mt * F(1 / 448)).astype(F) * F(0.9)).astype(F).reshape(-1)
    sv = ((vt * F(1 / 1.875)).astype(F) * F(0.999)).astype(F).reshape(-1)
    return w64, codes_m, sm, codes_v.astype(np.uint8), sv


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,offset", [(1, 0), (31, 1), (256, 0), (300, 0), (4096, 1), (4352, 0), (50_021, 0), (50_021, 3)])
def test_fold_apply8_is_the_formula_operation_by_operation(n, offset, gdtype):
    """Several steps from zero state: codes and scales are exactly those of the formula in fp32;
    w is within 2e-7*(|w| + lr): one rounding of w and 3 ulp on an update of at most a few lr."""
    opt = adama.AdamA()
    opt.set_weight_decay(0.01)
    w0 = wl.normal((n,), 0.02, torch.float32, 9)
    w = Guarded(n, offset=offset).fill(w0.cuda())
    copy = Guarded(n, dtype=torch.bfloat16, offset=offset).zero()
    raw = State8.zeros(n + 16)
    s = State8(raw.m_codes[offset:offset + n], raw.m_scale[:-(-n // 256)], raw.v_codes[offset:offset + n], raw.v_scale[:-(-n // 256)])
    spread = torch.exp(3 * wl.normal((n,), 1.0, torch.float32, 4))
    for step in range(4):
        g = (wl.normal((n,), 1e-3, torch.float32, 20 + step) * spread).to(gdtype)
        g[5::7] = 0
        gg = Guarded(n, dtype=gdtype, offset=offset).fill(g.cuda())
        factor = 0.5 + step
        want = _emulate_step8(w.view.cpu().numpy(), g.float().numpy(), s, step + 1, wl.LR, factor, 0.01)
        opt.begin_minibatch(1)
        opt.fold_apply8_multi([w.view], [gg.view], [s], wl.LR, w_bf16=[copy.view],
                              grad_factor=torch.full((1,), factor, device="cuda"))
        assert np.all(np.abs(f64(w.view) - want[0]) <= 2e-7 * (np.abs(want[0]) + wl.LR * 10))
        assert torch.equal(copy.view, w.view.bfloat16())
        assert np.array_equal(s.m_codes.view(torch.uint8).cpu().numpy() & 127, want[1] & 127)
        assert np.array_equal(s.m_scale.cpu().numpy(), want[2])
        assert np.array_equal(s.v_codes.cpu().numpy(), want[3])
        assert np.array_equal(s.v_scale.cpu().numpy(), want[4])
        for b in (w, copy, gg):
            b.check()
    assert not bool(raw.m_codes.view(torch.uint8)[offset + n:].any()) and not bool(raw.v_codes[offset + n:].any())


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 8, 1])
def test_long_8_bit_lists_equal_one_tensor_at_a_time(gdtype, offset):
    """A long list is streamed through shared memory, single tensors of up to a million elements are
    not: the same codes, scales and weights, whole blocks or ragged, aligned (offset 0 and 8 elements
    of 16 bytes) or element by element (offset 1)."""
    sizes = [1_000_000, 255, 256, 4097, 900_001, 3, 70_000]
    gen = torch.Generator(device="cuda").manual_seed(offset)
    off8 = 16 if offset == 8 else offset                        # codes are bytes
    ws = [Guarded(n, offset=offset) for n in sizes]
    gs = [Guarded(n, dtype=gdtype, offset=offset) for n in sizes]
    cs = [Guarded(n, dtype=torch.bfloat16, offset=offset) for n in sizes]
    for w, g in zip(ws, gs):
        w.view.copy_(torch.randn(w.n, generator=gen, device="cuda") * 0.02)
        g.view.copy_((torch.randn(w.n, generator=gen, device="cuda") * 1e-3).to(gdtype))
    w2 = [w.view.clone() for w in ws]

    def states():
        raw = [State8.zeros(n + 32) for n in sizes]
        return raw, [State8(r.m_codes[off8:off8 + n], r.m_scale[1:1 - (-n // 256)] if n + 32 > 256 * -(-n // 256) else
                            r.m_scale[:-(-n // 256)], r.v_codes[off8:off8 + n], r.v_scale[:-(-n // 256)]) for r, n in zip(raw, sizes)]

    raw1, s1 = states()
    raw2, s2 = states()
    a, b = adama.AdamA(), adama.AdamA()
    for step in range(3):
        a.begin_minibatch(1)
        b.begin_minibatch(1)
        a.fold_apply8_multi([w.view for w in ws], [g.view for g in gs], s1, wl.LR, w_bf16=[c.view for c in cs])
        for w, g, s in zip(w2, gs, s2):
            b.fold_apply8_multi([w], [g.view], [s], wl.LR)
    a.sync_status()
    assert a.launch_count == 3
    for w, y, c, g in zip(ws, w2, cs, gs):
        assert torch.equal(w.view, y) and torch.equal(c.view, y.bfloat16())
        for x in (w, c, g):
            x.check()
    for x, y in zip(raw1, raw2):      # the bytes around the states too: untouched zeros
        assert torch.equal(x.m_codes.view(torch.uint8), y.m_codes.view(torch.uint8)) and torch.equal(x.v_codes, y.v_codes)
        assert torch.equal(x.m_scale, y.m_scale) and torch.equal(x.v_scale, y.v_scale)
    ms, vs = [torch.empty(n, device="cuda") for n in sizes], [torch.empty(n, device="cuda") for n in sizes]
    a.state8_unpack_multi(s1, ms, vs)
    for s, m, v in zip(s1, ms, vs):
        dm, dv = _decode(s)
        assert np.array_equal(f64(m), dm.astype(F).astype(float)) and np.array_equal(f64(v), dv.astype(F).astype(float))


def test_fold_apply8_tracks_32_bit_states():
    """200 steps of a noisy quadratic from the same start (mean square distance 1): the 8-bit run
    ends about as low as the 32-bit one, and v follows (codes that never move would not)."""
    n, steps = 20_000, 200
    target = wl.normal((n,), 1.0, torch.float32, 1).cuda()
    scale = torch.exp(2 * wl.normal((n,), 1.0, torch.float32, 2)).cuda()
    ends = []
    for eight in (False, True):
        opt = adama.AdamA()
        w = torch.zeros(n, device="cuda")
        m, v, s = torch.zeros_like(w), torch.zeros_like(w), State8.zeros(n)
        for i in range(steps):
            g = scale * ((w - target) + wl.normal((n,), 0.1, torch.float32, 50 + i).cuda())
            opt.begin_minibatch(1)
            if eight:
                opt.fold_apply8_multi([w], [g], [s], 2e-2)
            else:
                opt.fold_apply_multi([w], [g], [m], [v], 2e-2)
        ends.append(float((w - target).square().mean()))
        if not eight:
            v32 = v
        else:
            um, uv = torch.empty_like(w), torch.empty_like(w)
            opt.state8_unpack_multi([s], [um], [uv])
    assert ends[1] <= 1.5 * ends[0] + 1e-2, ends
    assert 0.5 < float((uv.sqrt() / v32.sqrt()).median()) < 2.0


def test_zero_gradients_and_denormal_moments_keep_the_state_finite():
    n = 512
    opt = adama.AdamA()
    w = torch.ones(n, device="cuda")
    s = State8.zeros(n)
    opt.begin_minibatch(1)
    opt.fold_apply8_multi([w], [torch.zeros(n, device="cuda")], [s], wl.LR)
    assert bool((w == 1).all()) and not bool(s.m_scale.any()) and not bool(s.v_codes.any())
    g = torch.full((n,), 1e-21, device="cuda")        # v = 1e-45: the smallest numbers there are
    g[::2] = 1e-20
    for _ in range(3):
        opt.begin_minibatch(1)
        opt.fold_apply8_multi([w], [g], [s], wl.LR)
    m, v = torch.empty_like(w), torch.empty_like(w)
    opt.state8_unpack_multi([s], [m], [v])
    for t in (w, m, v):
        assert bool(torch.isfinite(t).all())


def test_a_nan_gradient_spoils_its_own_block_only():
    n = 1024
    opt = adama.AdamA()
    w, g = torch.ones(n, device="cuda"), torch.full((n,), 1e-3, device="cuda")
    g[300] = math.nan
    s = State8.zeros(n)
    opt.begin_minibatch(1)
    opt.fold_apply8_multi([w], [g], [s], wl.LR)
    m, v = torch.empty_like(w), torch.empty_like(w)
    opt.state8_unpack_multi([s], [m], [v])
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[256:512] = True
    assert torch.equal(torch.isnan(m), bad) and torch.equal(torch.isnan(v), bad)
    assert int(torch.isnan(w).sum()) == 1


def test_many_8_bit_tensors_in_several_launches_equal_one_by_one():
    sizes = [(53 * i) % 700 for i in range(900)]
    opt, ref = adama.AdamA(), adama.AdamA()
    ws = [wl.normal((n,), 0.02, torch.float32, i).cuda() for i, n in enumerate(sizes)]
    gs = [wl.normal((n,), 1e-3, torch.bfloat16, 9000 + i).cuda() for i, n in enumerate(sizes)]
    w2 = [w.clone() for w in ws]
    a, b = [State8.zeros(n) for n in sizes], [State8.zeros(n) for n in sizes]
    opt.begin_minibatch(1)
    ref.begin_minibatch(1)
    opt.fold_apply8_multi(ws, gs, State8List(a), wl.LR)
    assert opt.launch_count == 3                # at most 448 in a launch
    for w, g, s in zip(w2, gs, b):
        ref.fold_apply8_multi([w], [g], [s], wl.LR)
    for x, y in zip(ws, w2):
        assert torch.equal(x, y)
    for x, y in zip(a, b):
        assert torch.equal(x.m_scale, y.m_scale) and torch.equal(x.v_codes, y.v_codes)
        assert torch.equal(x.m_codes.view(torch.uint8), y.m_codes.view(torch.uint8))


@pytest.mark.parametrize("large", [0, 3_000_017])
@pytest.mark.parametrize("count", [64, 65, 192, 193])
def test_lists_around_the_sizes_of_the_launch_tables(count, large):
    """The same tensors in one list and one by one; with one large tensor in the list's middle they stream."""
    sizes = [1 + (53 * i) % 700 for i in range(count)]
    sizes[count // 2] += large
    lists = lambda: [[wl.normal((n,), 0.02, torch.float32, k * 1000 + i).cuda() for i, n in enumerate(sizes)]  # noqa: E731
                     for k in range(3)]
    gs = [wl.normal((n,), 1e-3, torch.bfloat16, 9000 + i).cuda() for i, n in enumerate(sizes)]
    opt, ref = adama.AdamA(), adama.AdamA()
    opt.begin_minibatch(1)
    ref.begin_minibatch(1)
    (w, m, v), (w2, m2, v2) = lists(), lists()
    v, v2 = [x.abs() for x in v], [x.abs() for x in v2]
    a, b = [State8.zeros(n) for n in sizes], [State8.zeros(n) for n in sizes]
    opt.state8_pack_multi(m, v, State8List(a))
    opt.fold_apply_multi(w, gs, m, v, wl.LR)
    opt.fold_apply8_multi(w, gs, State8List(a), wl.LR)
    m8, v8, m9, v9 = ([torch.full((n,), -1.0, device="cuda") for n in sizes] for _ in range(4))
    opt.state8_unpack_multi(State8List(a), m8, v8)
    for i in range(count):
        ref.state8_pack_multi([m2[i]], [v2[i]], [b[i]])
        ref.fold_apply_multi([w2[i]], [gs[i]], [m2[i]], [v2[i]], wl.LR)
        ref.fold_apply8_multi([w2[i]], [gs[i]], [b[i]], wl.LR)
        ref.state8_unpack_multi([b[i]], [m9[i]], [v9[i]])
    assert opt.launch_count == 4
    for x, y in zip(w + m + v + m8 + v8, w2 + m2 + v2 + m9 + v9):
        assert torch.equal(x, y)
    opt.sync_status()


def test_one_tensor_of_more_than_2_31_elements():
    """32-bit states (34 GB), then 8-bit ones in place of the moments: what lies around and behind element
    2^31 becomes what the same values become in tensors of their own; the norm counts every element."""
    n = 2 ** 31 + 12_345
    if torch.cuda.mem_get_info()[0] < 48 * 2 ** 30:
        pytest.skip("needs 48 GB of free device memory")
    parts = [slice(0, 4096), slice(2 ** 31 - 8192, 2 ** 31 + 4096), slice(2 ** 31 + 8192, n)]
    opt, ref = adama.AdamA(), adama.AdamA()
    opt.begin_minibatch(1)
    ref.begin_minibatch(1)
    g = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(4, device="cuda")
    opt.grad_norm_multi([g], 1.0, out)
    assert float(out[2:4].view(torch.float64)) == n
    w, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    for k, p in enumerate(parts):
        size = (p.stop - p.start,)
        for j, t in enumerate((w, m, v, g)):
            t[p] = wl.normal(size, 0.02, torch.float32, 10 * k + j).abs().cuda()
    small = [[t[p].clone() for t in (w, g, m, v)] for p in parts]
    opt.fold_apply_multi([w], [g], [m], [v], wl.LR)
    for p, (w1, g1, m1, v1) in zip(parts, small):
        ref.fold_apply_multi([w1], [g1], [m1], [v1], wl.LR)
        assert torch.equal(w[p], w1) and torch.equal(m[p], m1) and torch.equal(v[p], v1)
    state = State8.zeros(n)
    opt.state8_pack_multi([m], [v], [state])
    opt.fold_apply8_multi([w], [g], [state], wl.LR)
    opt.state8_unpack_multi([state], [m], [v])
    for p, (w1, g1, m1, v1) in zip(parts, small):
        one = State8.zeros(w1.numel())
        ref.state8_pack_multi([m1], [v1], [one])
        ref.fold_apply8_multi([w1], [g1], [one], wl.LR)
        ref.state8_unpack_multi([one], [m1], [v1])
        assert torch.equal(w[p], w1) and torch.equal(m[p], m1) and torch.equal(v[p], v1)
    opt.sync_status()


# ---- gradient norm ---------------------------------------------------------------------------------

@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes,offset", [([1], 0), ([3, 1, 2], 1), ([4096, 5, 0, 4097], 3), ([100_003, 17], 1),
                                          ([(31 * i) % 200 for i in range(2100)], 1), ([3_000_001], 0)])
def test_grad_norm_against_64_bits(sizes, offset, gdtype):
    """Squares and sums of up to 64 elements in fp32 (13 roundings at most), the rest in double: relative
    error of the sum <= 1.0e-6 (17*2^-24), half of it on the norm, one more rounding on the factor."""
    opt = adama.AdamA()
    gs = _views(sizes, offset, gdtype)
    for i, g in enumerate(gs):
        g.copy_(wl.normal((g.numel(),), 1e-2, torch.float32, 40 + i))
    want = math.sqrt(sum(float((f64(g) ** 2).sum()) for g in gs))
    out = torch.full((4,), -1.0, device="cuda")
    for max_norm in (0.25 * want, 4 * want):
        opt.grad_norm_multi(gs, max_norm, out)
        first = out.clone()
        opt.grad_norm_multi(gs, max_norm, out)
        assert torch.equal(first, out)                                   # deterministic, workspace ready again
        assert abs(float(out[0]) - want) <= 6e-7 * want
        assert abs(float(out[1]) - min(1.0, max_norm / want)) <= 7e-7
        assert abs(float(out[2:4].view(torch.float64)) - want * want) <= 1.1e-6 * want * want


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
def test_grad_norm_counts_every_element_once(gdtype):
    """Of ones, whose sums are exact at any order, at every alignment and around the lengths where a tensor
    ends near the 32 KB that one thread block takes at a time."""
    opt = adama.AdamA()
    chunk = 32768 // (2 if gdtype == torch.bfloat16 else 4)
    x = torch.ones(2 * chunk + 64, dtype=gdtype, device="cuda")
    out = torch.zeros(4, device="cuda")
    for n in [*range(1, 20), *range(chunk - 9, chunk + 10), *range(2 * chunk - 9, 2 * chunk + 10)]:
        for offset in range(8):
            x.fill_(math.nan)
            x[offset:offset + n] = 1
            opt.grad_norm_multi([x[offset:offset + n]], 1.0, out)
            assert float(out[2:4].view(torch.float64)) == n, (n, offset)


def test_grad_norm_joins_lists_and_reports_what_is_not_finite():
    opt = adama.AdamA()
    a, b = wl.normal((5000,), 1.0, torch.float32, 1).cuda(), wl.normal((777,), 1.0, torch.bfloat16, 2).cuda()
    out = torch.zeros(4, device="cuda")
    opt.grad_norm_multi([a], 1.0, out)
    opt.grad_norm_multi([b], 1.0, out, accumulate=True)
    want = math.sqrt(float((f64(a) ** 2).sum() + (f64(b) ** 2).sum()))
    assert abs(float(out[0]) - want) <= 6e-7 * want
    opt.grad_norm_multi([], 1.0, out)
    assert out[:2].tolist() == [0.0, 1.0]
    for bad in (math.inf, -math.inf, math.nan):
        a[4321] = bad
        opt.grad_norm_multi([a, a[:100]], 1.0, out)
        assert not math.isfinite(float(out[0])) and math.isnan(float(out[1]))
    a[4321] = 0
    with pytest.raises(TypeError):
        opt.grad_norm_multi([a, b], 1.0, out)             # one dtype per call
    opt.grad_norm_multi([a], math.inf, out)
    assert float(out[1]) == 1.0


def test_step_calls_on_another_stream():
    n = 300_000
    s = torch.cuda.Stream()
    opt = adama.AdamA()
    w = wl.normal((n,), 0.02, torch.float32, 1).cuda()
    g = wl.normal((n,), 1e-2, torch.bfloat16, 2).cuda()
    w2, st, st2, out = w.clone(), State8.zeros(n), State8.zeros(n), torch.empty(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(3):
            opt.begin_minibatch(1)
            opt.grad_norm_multi([g], 1.0, out)
            opt.fold_apply8_multi([w], [g], [st], wl.LR, grad_factor=out[1:2])
    s.synchronize()
    ref = adama.AdamA()
    for _ in range(3):
        ref.begin_minibatch(1)
        ref.fold_apply8_multi([w2], [g], [st2], wl.LR, grad_factor=out[1:2])
    assert torch.equal(w, w2) and torch.equal(st.v_codes, st2.v_codes)


def test_step_refusals():
    opt = adama.AdamA()
    f = lambda n, dt=torch.float32: torch.zeros(n, dtype=dt, device="cuda")  # noqa: E731
    x = f(8)

    def err(fn, *a, **k):
        with pytest.raises(adama.AdamAError) as e:
            fn(*a, **k)
        return e.value.status

    assert err(opt.fold_apply_multi, [x], [f(8)], [f(8)], [f(8)], 1e-3) == Status.ERR_BAD_STATE
    assert err(opt.fold_apply8_multi, [x], [f(8)], [State8.zeros(8)], 1e-3) == Status.ERR_BAD_STATE
    opt.begin_minibatch(1)
    assert err(opt.fold_apply_multi, [x], [f(8)], [f(8)], [f(8)], math.nan) == Status.ERR_INVALID_ARG
    assert err(opt.grad_norm_multi, [x], 0.0, f(4)) == Status.ERR_INVALID_ARG
    assert err(opt.grad_norm_multi, [x], math.nan, f(4)) == Status.ERR_INVALID_ARG
    assert err(opt.grad_norm_multi, [x], 1.0, f(8)[1:5]) == Status.ERR_MISALIGNED
    with pytest.raises(ValueError):
        opt.fold_apply_multi([x], [f(7)], [f(8)], [f(8)], 1e-3)
    with pytest.raises(ValueError):
        opt.fold_apply8_multi([x], [f(8)], [State8.zeros(9)], 1e-3)
    with pytest.raises(ValueError):
        opt.fold_apply_multi([x], [f(8)], [f(8)], [f(8)], 1e-3, w_bf16=[f(7, torch.bfloat16)])
    with pytest.raises(ValueError):
        opt.fold_apply_multi([x], [f(8)], [f(8)], [f(8)], 1e-3, grad_factor=f(2))
    with pytest.raises(TypeError):
        opt.fold_apply_multi([x], [f(8, torch.float16)], [f(8)], [f(8)], 1e-3)
    with pytest.raises(TypeError):
        opt.fold_apply_multi([x], [f(8)], [f(8)], [f(8)], 1e-3, w_bf16=[f(8)])
    with pytest.raises(TypeError):
        opt.fold_apply_multi([x], [f(8)], [f(8)], [f(8)], 1e-3, grad_factor=torch.ones(1))
    with pytest.raises(TypeError):
        State8(f(8, torch.uint8), f(1), f(8, torch.uint8), f(1))
    with pytest.raises(ValueError):
        State8(f(257, torch.float8_e4m3fn), f(1), f(257, torch.uint8), f(2))
    opt.fold_apply_multi([], [], [], [], 1e-3)           # nothing to do
    opt.fold_apply_multi([f(0)], [f(0)], [f(0)], [f(0)], 1e-3)
    opt.fold_apply8_multi([], [], [], 1e-3)
    assert opt.launch_count == 0
    assert not bool(x.any())


def test_null_pointers_are_refused():
    """Through the C ABI: a null entry with elements behind it, a null list."""
    import ctypes
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    L, x = adama.load_library(), torch.zeros(8, device="cuda")
    ptr, none = (ctypes.c_void_p * 1)(x.data_ptr()), (ctypes.c_void_p * 1)(None)
    odd = (ctypes.c_void_p * 1)(x.data_ptr() + 2)
    n = (ctypes.c_size_t * 1)(8)
    call = lambda g, w, m, v, cnt=1: L.adama_fold_apply_multi(opt._h, g, 0, w, m, v, None, n, cnt, 1e-3, None, None)  # noqa: E731
    assert call(none, ptr, ptr, ptr) == Status.ERR_INVALID_ARG
    assert call(ptr, none, ptr, ptr) == Status.ERR_INVALID_ARG
    assert call(ptr, ptr, None, ptr) == Status.ERR_INVALID_ARG
    assert call(ptr, ptr, ptr, ptr, -1) == Status.ERR_INVALID_ARG
    assert call(ptr, ptr, ptr, odd) == Status.ERR_MISALIGNED
    assert L.adama_fold_apply8_multi(opt._h, ptr, 0, ptr, None, None, n, 1, 1e-3, None, None) == Status.ERR_INVALID_ARG
    assert L.adama_grad_norm_multi(opt._h, ptr, 0, n, 1, 1.0, 0, None, x.data_ptr(), None) == Status.ERR_INVALID_ARG
    assert L.adama_grad_norm_multi(opt._h, ptr, 0, n, 1, 1.0, 0, x.data_ptr(), None, None) == Status.ERR_INVALID_ARG
    assert opt.launch_count == 0
