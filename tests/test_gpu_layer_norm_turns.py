"""Layer norm and its backward pass with many rows to a block: every group of warps goes round at least four times (of 148 SMs), so that
what rows lie in is used again, in all types, for even and uneven rows.  Formulas in 64 bits; tolerances, u = 2^-24, as for
few rows but for the sums over rows: a thread adds the rows of its block one after the other, then the groups of a block (16 at
most), then 16 warps take every 16th of the blocks' sums and add theirs: (R/B + 16 + B/16 + 16 + 4)*u*sum|.|, with B blocks of rows
and 4 for a row's own product.  B is at least min(R, SMs) for up to 8192 columns and at least ceil(4*SMs/tiles) for more, where a tile
has 512 columns."""
import pytest
import torch

import paper_2305_19982_b200 as adama
from test_gpu_layer_norm import TYPES, U, _check, _inputs, _K, _matrix, _outside_untouched, _reference_back

pytestmark = pytest.mark.gpu


def _blocks(R, D):
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles = -(-D // 512)
    return min(R, sms if D <= 8192 else -(-4 * sms // tiles))


def _sum_bound(R, D):
    B = _blocks(R, D)
    return (-(-R // B) + 16 + -(-B // 16) + 16 + 4) * U


def _compare(opt, x, dy, w, b, y, dx, mean, rstd):
    R, D = x.shape
    dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd, eps=1e-5)
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    K = _K(D)
    for at in range(0, R, 2000):                          # (in pieces: 64 bits take room)
        rows = slice(at, at + 2000)
        x64 = x[rows].double()
        rmean = x64.mean(1, keepdim=True)
        rrstd = ((x64 - rmean).square().mean(1, keepdim=True) + 1e-5) ** -0.5
        size, xhat = x64.abs().mean(1, keepdim=True), (x64 - rmean) * rrstd
        # the mean's error moves every x - mean alike: it adds its square to the variance, or rounds the largest of them
        spread = K + 4 * U + K * size * rrstd * U + (K * size * rrstd) ** 2
        tol = w.double().abs() * (xhat.abs() * spread + rrstd * K * size) + 4 * U * ((w * xhat).abs() + b.double().abs())
        _check(y[rows], xhat * w.double() + b.double(), tol, y.dtype, "y")
        _check(mean[rows], rmean[:, 0], K * size[:, 0], torch.float32, "mean")
        _check(rstd[rows], rrstd[:, 0], spread[:, 0] * rrstd[:, 0], torch.float32, "rstd")
        rdx, tdx = _reference_back(dy[rows], x[rows], w, mean[rows], rstd[rows])[:2]
        _check(dx[rows], rdx, tdx, dx.dtype, "dx")
    terms = [torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(4)]
    for at in range(0, R, 2000):
        rows = slice(at, at + 2000)
        dy64 = dy[rows].double()
        products = dy64 * ((x[rows].double() - mean[rows, None].double()) * rstd[rows, None].double())
        for total, part in zip(terms, (products, products.abs(), dy64, dy64.abs())):
            total += part.sum(0)
    _check(dw, terms[0], _sum_bound(R, D) * terms[1], torch.float32, "dweight")
    _check(db, terms[2], _sum_bound(R, D) * terms[3], torch.float32, "dbias")
    return dw, db


# lanes to a row; one to sixteen warps to a row, one or several groups to a block, one and two pieces of a thread
SHAPES = [(80_003, 24), (19_001, 100), (9601, 252), (9601, 300), (9601, 512), (9601, 1004), (9601, 1600), (9601, 1601), (4801, 2500), (4801, 4096),
          (2401, 6152), (2401, 8192), (2401, 8191)]


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("R,D", SHAPES)
@pytest.mark.parametrize("pitch,offset", [(0, 0), (3, 1)])
def test_many_turns(R, D, xt, yt, pitch, offset):
    opt = adama.AdamA()
    (_, x), (_, dy), w, b = _inputs(R, D, xt, yt, pitch, offset, R + D)
    (ybuf, y), (dxbuf, dx) = _matrix(R, D, yt, pitch, offset), _matrix(R, D, xt, pitch, offset)
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    sums = _compare(opt, x, dy, w, b, y, dx, mean, rstd)
    _outside_untouched(ybuf, y)
    _outside_untouched(dxbuf, dx)
    first = y.clone(), dx.clone()
    for _ in range(3):                                    # bit for bit
        y.fill_(7.0)
        dx.fill_(7.0)
        dw, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
        opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
        opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
        assert all(torch.equal(p, q) for p, q in zip((y, dx, dw, db), first + sums))
    opt.sync_status()


@pytest.mark.parametrize("xt,yt", TYPES)
@pytest.mark.parametrize("R,D", [(3000, 8200), (2500, 12_288), (2000, 16_401), (300, 40_001)])
def test_many_rows_that_no_group_holds(R, D, xt, yt):
    opt = adama.AdamA()
    (_, x), (_, dy), w, b = _inputs(R, D, xt, yt, 0, 0, R + D)
    y, dx = torch.empty(R, D, dtype=yt, device="cuda"), torch.empty(R, D, dtype=xt, device="cuda")
    mean, rstd = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    _compare(opt, x, dy, w, b, y, dx, mean, rstd)
    opt.sync_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,D", [(19_001, 100), (9601, 1004), (9601, 1600), (9601, 1601), (2401, 6152)])
def test_many_turns_in_place(R, D, dtype):
    opt = adama.AdamA()
    (_, x), (_, dy), w, b = _inputs(R, D, dtype, dtype, 0, 0, R + D)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    opt.layer_norm(x, w, b, y, mean=mean, rstd=rstd)
    opt.layer_norm_backward(dy, x, w, mean, rstd, dx)
    over = x.clone()
    opt.layer_norm(over, w, b, over)
    assert torch.equal(over, y)
    for which in range(2):
        a = [dy.clone(), x.clone()]
        opt.layer_norm_backward(a[0], a[1], w, mean, rstd, a[which])
        assert torch.equal(a[which], dx)
