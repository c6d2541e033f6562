"""Layer norm (adama_layer_norm) and its backward pass (adama_layer_norm_backward) against the formulas in 64 bits.

Tolerances, u = 2^-24.  A sum over a row of D elements passes through at most 8*ceil(D/4096) + 3 additions in a thread, 5 between lanes
and 16 over warps: its error is at most K = (8*ceil(D/4096) + 24)*u of the mean magnitude.
    y: mean K*mean|x|, rstd relative K, the operations behind them 4u: |w|*(|xhat|*(K + 4u) + rstd*K*mean|x|) + 4u*(|w xhat| + |b|)
    dx: rstd*(K*(mean|g| + |xhat|*mean|g xhat|) + 8u*(|g| + |s1| + |xhat s2|))   (mean and rstd are inputs)
    dweight, dbias: a thread adds its block's rows one after the other (R/64 of them at most, where blocks are fewer than rows), then
        come at most 16 sums in a block, 19 of blocks and 16 of these: (R/64 + 64)*u*sum|.|
and half a last place of the output's type each."""
import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]
SENTINEL = 777.0


def _matrix(rows, cols, dtype, pitch=0, offset=0, values=None):
    """(buffer, [rows, cols] view of it) with `pitch` elements between rows, `offset` in front, sentinels around."""
    ld = cols + pitch
    buf = torch.full((offset + rows * ld + 64,), SENTINEL, dtype=dtype, device="cuda")
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    if values is not None:
        view.copy_(values)
    return buf, view


def _outside_untouched(buf, view):
    mask = torch.ones_like(buf, dtype=torch.bool)
    at = view.storage_offset() - buf.storage_offset()
    inner = mask[at:at + view.shape[0] * view.stride(0)] if view.shape[0] else mask[:0]
    if view.shape[0]:
        inner.view(view.shape[0], view.stride(0))[:, :view.shape[1]] = False
    assert bool((buf[mask] == SENTINEL).all())


def _inputs(R, D, xt, yt, pitch, offset, seed):
    n = lambda shape, std, k: wl.normal(shape, std, torch.float32, seed + k, device="cuda")  # noqa: E731
    x = _matrix(R, D, xt, pitch, offset, n((R, D), 1.5, 0) + 4 * n((R, 1), 1.0, 1))
    dy = _matrix(R, D, yt, pitch, (offset * 3) % 8, n((R, D), 1e-2, 2))
    return x, dy, 1 + 0.2 * n((D,), 1.0, 3), 0.3 * n((D,), 1.0, 4)


def _K(D):
    return (8 * -(-D // 4096) + 24) * U


def _check(got, want, tol, dtype, what):
    err = (got.double() - want).abs()
    assert bool((err <= tol + HALF_ULP[dtype] * want.abs()).all()), f"{what}: {float((err - tol).max())}"


def _reference_back(dy, x, w, mean, rstd):
    dy, x, w, mean, rstd = dy.double(), x.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    xhat, g = (x - mean) * rstd, dy * w
    s1, s2 = g.mean(1, keepdim=True), (g * xhat).mean(1, keepdim=True)
    D, R = x.shape[1], x.shape[0]
    K = _K(D)
    tol = rstd * (K * (g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
                  + 8 * U * (g.abs() + s1.abs() + (xhat * s2).abs()))
    rows = (R / 64 + 64) * U
    return (rstd * (g - s1 - xhat * s2), tol, (dy * xhat).sum(0), rows * (dy * xhat).abs().sum(0), dy.sum(0), rows * dy.abs().sum(0))


SHAPES = [(1, 1), (3, 2), (1, 7), (9, 8), (70, 9), (33, 31), (300, 64), (5, 257), (2, 1600), (301, 1000), (7, 1601), (40, 4099), (3, 8192),
          (3, 8193), (2, 16384), (2, 16390), (65, 16401), (9, 4), (70, 12), (33, 260), (301, 1004), (40, 4100), (300, 6152), (2, 8188)]


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("R,D", SHAPES)
@pytest.mark.parametrize("pitch,offset", [(0, 0), (3, 1), (8, 5)])
def test_layer_norm_and_its_backward_pass(R, D, xt, yt, pitch, offset):
    opt = adama.AdamA()
    (xbuf, x), (dybuf, dy), w, b = _inputs(R, D, xt, yt, pitch, offset, R + D)
    ybuf, y = _matrix(R, D, yt, pitch + 1, offset)
    mean, rstd = (torch.full((R,), SENTINEL, device="cuda") for _ in range(2))
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd, eps=1e-5)
    x64, K = x.double(), _K(D)
    rmean = x64.mean(1, keepdim=True)
    rrstd = ((x64 - rmean).square().mean(1, keepdim=True) + 1e-5) ** -0.5
    size = x64.abs().mean(1, keepdim=True)
    xhat = (x64 - rmean) * rrstd
    # the mean's error moves every x - mean alike: it adds its square to the variance, or rounds the largest of them
    spread = K + 4 * U + K * size * rrstd * U + (K * size * rrstd) ** 2
    want = xhat * w.double() + b.double()
    tol = w.double().abs() * (xhat.abs() * spread + rrstd * K * size) + 4 * U * ((w * xhat).abs() + b.double().abs())
    _check(y, want, tol, yt, "y")
    _check(mean, rmean[:, 0], K * size[:, 0], torch.float32, "mean")
    _check(rstd, rrstd[:, 0], spread[:, 0] * rrstd[:, 0], torch.float32, "rstd")
    _outside_untouched(ybuf, y)

    dxbuf, dx = _matrix(R, D, xt, pitch, (offset * 5) % 8)
    dw, db = (torch.full((D,), SENTINEL, device="cuda") for _ in range(2))
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    rdx, tdx, rdw, tdw, rdb, tdb = _reference_back(dy, x, w, mean, rstd)
    _check(dx, rdx, tdx, xt, "dx")
    _check(dw, rdw, tdw, torch.float32, "dweight")
    _check(db, rdb, tdb, torch.float32, "dbias")
    _outside_untouched(dxbuf, dx)
    again = torch.empty_like(dw), torch.empty_like(db)
    opt.layer_norm_backward(dy, x, w, mean, rstd, None, *again)        # without dx: the same sums
    assert torch.equal(again[0], dw) and torch.equal(again[1], db)
    only = torch.empty_like(dx)
    opt.layer_norm_backward(dy, x, w, mean, rstd, only)                # dx alone
    assert torch.equal(only, dx)
    opt.sync_status()


@pytest.mark.parametrize("R,D", [(100_003, 24), (2000, 100), (4096, 1600), (1024, 4096), (513, 8200)])
def test_many_rows(R, D):
    """Several turns of every block, and sums over many blocks."""
    opt = adama.AdamA()
    (_, x), (_, dy), w, b = _inputs(R, D, torch.bfloat16, torch.bfloat16, 0, 0, 7)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    rdx, tdx, rdw, tdw, rdb, tdb = _reference_back(dy, x, w, mean, rstd)
    _check(dx, rdx, tdx, torch.bfloat16, "dx")
    _check(dw, rdw, tdw, torch.float32, "dweight")
    _check(db, rdb, tdb, torch.float32, "dbias")
    first = dx.clone(), dw.clone(), db.clone()
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    assert all(torch.equal(p, q) for p, q in zip(first, (dx, dw, db)))  # bit for bit


@pytest.mark.parametrize("R,D", [(1, 5), (37, 200), (64, 1600), (3, 9001)])
def test_parameters_gradients_folded_into_moments(R, D):
    """As adama_fold does it with the gradients that the other form writes, bit for bit."""
    opt = adama.AdamA()
    opt.begin_minibatch(4)
    (_, x), (_, dy), w, _ = _inputs(R, D, torch.float32, torch.bfloat16, 0, 0, 3)
    mean, rstd = x.mean(1), 1 / x.std(1, correction=0)
    dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    dx, dx2 = torch.empty_like(x), torch.empty_like(x)
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    start = [wl.normal((D,), 1e-3, torch.float32, k, device="cuda") for k in range(4)]
    start[1], start[3] = start[1].square(), start[3].square()
    want, got = [t.clone() for t in start], [t.clone() for t in start]
    opt.fold(dw, want[0], want[1])
    opt.fold(db, want[2], want[3])
    opt.layer_norm_backward_fold(dy, x, w, mean, rstd, dx2, *got)
    assert torch.equal(dx, dx2) and all(torch.equal(p, q) for p, q in zip(got, want))
    weight_only = [t.clone() for t in start[:2]]
    opt.layer_norm_backward_fold(dy, x, w, mean, rstd, None, *weight_only)
    assert all(torch.equal(p, q) for p, q in zip(weight_only, want))


def test_without_a_bias_and_without_saved_statistics():
    opt = adama.AdamA()
    x, w = wl.normal((13, 300), 1.0, torch.float32, 1).cuda(), wl.normal((300,), 1.0, torch.float32, 2).cuda()
    y, z = torch.empty_like(x), torch.empty_like(x)
    opt.layer_norm(x, w, None, y)
    opt.layer_norm(x, w, torch.zeros(300, device="cuda"), z)
    assert torch.equal(y, z)


@pytest.mark.parametrize("D", [24, 200, 1600, 1603, 9000, 17_001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place(D, dtype):
    opt = adama.AdamA()
    R = 50
    x, dy = (wl.normal((R, D), s, torch.float32, 5).cuda().to(dtype) for s in (1.0, 1e-2))
    w, b = wl.normal((D,), 1.0, torch.float32, 6).cuda(), wl.normal((D,), 1.0, torch.float32, 7).cuda()
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    over = x.clone()
    opt.layer_norm(over, w, b, over)
    assert torch.equal(over, y)
    for which in range(2):
        a, c = dy.clone(), x.clone()
        dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
        opt.layer_norm_backward(a, c, w, mean, rstd, (a, c)[which], dw2, db2)
        assert torch.equal((a, c)[which], dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_no_rows():
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    x, w, none = torch.empty(0, 40, device="cuda"), torch.ones(40, device="cuda"), torch.empty(0, device="cuda")
    opt.layer_norm(x, w, w, torch.empty_like(x), mean=none, rstd=none)
    dw, db = torch.full((40,), SENTINEL, device="cuda"), torch.full((40,), SENTINEL, device="cuda")
    opt.layer_norm_backward(x, x, w, none, none, torch.empty_like(x), dw, db)
    assert float(dw.abs().max()) == 0 and float(db.abs().max()) == 0
    m, v = torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    opt.layer_norm_backward_fold(x, x, w, none, none, None, m, v)
    assert bool((m == 1).all()) and bool((v == 1).all())
    opt.sync_status()


def test_a_common_offset_and_a_constant_row():
    """Rows of 4096 + small steps (exact in fp32): the offset cancels before anything is squared.  A row of one value
    has variance 0 and gives the bias."""
    opt = adama.AdamA()
    base = (torch.randint(-64, 65, (4, 1000), generator=torch.Generator().manual_seed(1)) / 64.0).cuda()
    w, b = torch.ones(1000, device="cuda"), torch.full((1000,), 0.25, device="cuda")
    y, z = torch.empty_like(base), torch.empty_like(base)
    opt.layer_norm(base, w, b, y)
    opt.layer_norm(base + 4096, w, b, z)
    # the mean of the shifted rows is rounded at 4096: 2^-12, its sum's error K*4096 more
    assert float((y - z).abs().max()) <= 2 * (2.0 ** -12 + _K(1000) * 4096) / float(base.std(1, correction=0).min())
    opt.layer_norm(torch.full((4, 1000), 3.0, device="cuda"), w, b, y)
    assert bool((y == 0.25).all())


def test_a_row_that_is_not_finite_stays_alone():
    opt = adama.AdamA()
    x = wl.normal((40, 72), 1.0, torch.float32, 1).cuda()
    w = torch.ones(72, device="cuda")
    y, clean = torch.empty_like(x), torch.empty_like(x)
    opt.layer_norm(x, w, w, clean)
    x[3, 5], x[17, 0] = float("nan"), float("inf")
    opt.layer_norm(x, w, w, y)
    rest = [i for i in range(40) if i not in (3, 17)]
    assert torch.isnan(y[3]).all() and torch.isnan(y[17]).all() and torch.equal(y[rest], clean[rest])


def test_gradient_against_differences():
    """d(sum dy*y)/dx, /dweight, /dbias by central differences of the 64-bit formula."""
    opt = adama.AdamA()
    R, D = 3, 11
    x, dy = wl.normal((R, D), 1.0, torch.float32, 1).cuda(), wl.normal((R, D), 1.0, torch.float32, 2).cuda()
    w, b = wl.normal((D,), 1.0, torch.float32, 3).cuda(), wl.normal((D,), 1.0, torch.float32, 4).cuda()
    y, mean, rstd = torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)

    def loss(x, w, b):
        mean = x.mean(1, keepdims=True)
        return float(((x - mean) / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + 1e-5) * w + b).ravel() @ dy.double().cpu().numpy().ravel())

    args = [t.double().cpu().numpy() for t in (x, w, b)]
    for which, grad in enumerate((dx, dw, db)):
        for at in np.ndindex(args[which].shape):
            plus, minus = [a.copy() for a in args], [a.copy() for a in args]
            plus[which][at] += 1e-5
            minus[which][at] -= 1e-5
            slope = (loss(*plus) - loss(*minus)) / 2e-5
            # differences: h^2 of the third derivative (1e-9) and 1e-16*|loss|/h (1e-10); the kernel 1e-5 of sums of some ten
            assert abs(float(grad[at]) - slope) <= 1e-4


def test_refusals():
    opt = adama.AdamA()
    x, w, r = torch.ones(4, 16, device="cuda"), torch.ones(16, device="cuda"), torch.ones(4, device="cuda")
    y = torch.empty_like(x)

    def refused(kind, call, *args, **kw):
        with pytest.raises(kind) as e:
            call(*args, **kw)
        return e.value

    norm, back, fold = opt.layer_norm, opt.layer_norm_backward, opt.layer_norm_backward_fold
    refused(ValueError, norm, x, w, w, torch.empty(4, 15, device="cuda"))
    refused(ValueError, norm, x, w[:15], w, y)
    refused(ValueError, norm, x.t(), w[:4], None, torch.empty(16, 4, device="cuda"))
    refused(TypeError, norm, x.half(), w, w, y)
    refused(TypeError, norm, x, w.bfloat16(), w, y)
    refused(TypeError, norm, x.cpu(), w, w, y)
    for eps in (-1.0, float("nan"), float("inf")):
        assert refused(adama.AdamAError, norm, x, w, w, y, eps=eps).status == Status.ERR_INVALID_ARG
    assert refused(adama.AdamAError, norm, x, None, w, y).status == Status.ERR_INVALID_ARG
    buf = torch.ones(80, device="cuda")
    assert refused(adama.AdamAError, norm, buf[:64].view(4, 16), w, w, buf.as_strided((4, 16), (17, 1))).status == Status.ERR_INVALID_ARG
    refused(ValueError, back, x, x, w, r, r[:3], y)
    refused(TypeError, back, x, x, w, r, r, y.bfloat16())
    refused(ValueError, back, x[:3], x, w, r, r, y)
    assert refused(adama.AdamAError, fold, x, x, w, r, r, y, w, w).status == Status.ERR_BAD_STATE
    opt.begin_minibatch(1)
    assert refused(adama.AdamAError, fold, x, x, w, r, r, y, w, w, w, None).status == Status.ERR_INVALID_ARG
    opt.sync_status()
