"""Embedding lookup (adama_embedding) and its gradient by sorted tokens (adama_embedding_grad) against the
definitions in 64 bits.

Tolerances, u = 2^-24: the lookup is one product (u) and one rounding to the output's type.  A sum of n
vectors, in whatever groups, is off by at most n*u of the sum of the magnitudes, the scale adds u; a folded m by
a times that and u of itself, a folded v by b*(2|G| + e)*e and 3u of itself."""
import math

import numpy as np
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
SENTINEL = 777.0
TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)]


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


def _ids(T, V, kind, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "even":
        return torch.randint(0, V, (T,), generator=g).cuda()
    if kind == "one":                                   # a single token, all over
        return torch.full((T,), V // 2, dtype=torch.int64).cuda()
    if kind == "sorted":
        return torch.randint(0, V, (T,), generator=g).sort().values.cuda()
    if kind == "distinct":
        return torch.randperm(max(T, V), generator=g)[:T].remainder(V).cuda()
    ids = (V ** torch.rand(T, generator=g)).long().clamp(max=V) - 1   # "text": few tokens often
    if kind == "padded":
        ids[torch.rand(T, generator=g) < 0.3] = -1
    return ids.cuda()


def _sums(ids, dy, V, scale):
    """G, and the bound of its error, in float64."""
    live = ids >= 0
    n = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, ids[live], torch.ones_like(ids[live], dtype=torch.float64))
    add = lambda x: torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids[live], x[live].double())  # noqa: E731
    G = add(dy) * scale
    return G, (n[:, None] + 1) * U * add(dy.abs()) * abs(scale), n > 0


SHAPES = [(1, 1, 1), (1, 5, 7), (3, 2, 8), (9, 100, 9), (32, 11, 256), (33, 1000, 257), (131, 1003, 250), (200, 40, 1600), (700, 5000, 1601), (1500, 37, 33), (33, 50, 4), (131, 1003, 252), (200, 40, 1028)]


@pytest.mark.parametrize("tt,ot", TYPES)
@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("pitch,offset,scale", [(0, 0, 1.0), (3, 1, 11.3), (8, 5, -0.5)])
def test_lookup(T, V, D, tt, ot, pitch, offset, scale):
    opt = adama.AdamA()
    _, table = _matrix(V, D, tt, pitch, offset, wl.normal((V, D), 1.0, torch.float32, V, device="cuda"))
    ids = _ids(T, V, "padded", T)
    buf, out = _matrix(T, D, ot, pitch + 2, offset)
    opt.embedding(ids, table, out, scale=scale)
    s32 = float(torch.tensor(scale, dtype=torch.float32))
    want = torch.where(ids[:, None] >= 0, table[ids.clamp(min=0)].double() * s32, 0.0)
    assert bool(((out.double() - want).abs() <= (U + HALF_ULP[ot]) * want.abs()).all())
    if scale == 1.0 and tt == ot:
        assert torch.equal(out, torch.where(ids[:, None] >= 0, table[ids.clamp(min=0)], 0.0))
    _outside_untouched(buf, out)
    opt.sync_status()


@pytest.mark.parametrize("gt,dt", TYPES)
@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("kind,pitch,offset", [("text", 0, 0), ("padded", 3, 1), ("one", 8, 5)])
def test_gradient(T, V, D, gt, dt, kind, pitch, offset):
    opt = adama.AdamA()
    _, dy = _matrix(T, D, dt, pitch, offset, wl.normal((T, D), 1.0, torch.float32, T + V, device="cuda"))
    ids = _ids(T, V, kind, T + 1)
    G, tol, seen = _sums(ids, dy, V, 0.75)
    buf, grad = _matrix(V, D, gt, pitch + 2, (3 * offset) % 8)
    opt.embedding_grad(ids, dy, grad, scale=0.75)
    assert bool(((grad.double() - G).abs() <= tol + HALF_ULP[gt] * (G.abs() + tol)).all())
    assert bool((grad[~seen] == 0).all())
    _outside_untouched(buf, grad)
    start = wl.normal((V, D), 1.0, torch.float32, V + 1, device="cuda").to(gt)
    grad.copy_(start)
    opt.embedding_grad(ids, dy, grad, scale=0.75, accumulate=True)
    want = start.double() + G
    assert bool(((grad.double() - want).abs() <= tol + (HALF_ULP[gt] + U) * (want.abs() + tol)).all())
    assert torch.equal(grad[~seen], start[~seen])
    _outside_untouched(buf, grad)
    opt.sync_status()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,D,kind", [(1, 3, 5, "text"), (77, 50, 257, "padded"), (900, 2000, 1600, "text"), (3000, 999, 301, "one"), (3000, 999, 300, "one"), (500, 60, 1028, "text"), (64, 64, 8, "distinct"),
                                        (8192, 600, 24, "text"), (8193, 600, 24, "text")])
def test_folded_into_moments(T, V, D, kind, dt):
    opt = adama.AdamA()
    opt.begin_minibatch(4)
    a, b = (float(c) for c in adama.host_constants(0.9, 0.999, 1e-8, 4, 1, 1e-3)[:2])
    dy, ids = wl.normal((T, D), 1.0, torch.float32, 1, device="cuda").to(dt), _ids(T, V, kind, 2)
    G, e, seen = _sums(ids, dy, V, 2.5)
    mb, m = _matrix(V, D, torch.float32, 5, 3, wl.normal((V, D), 0.1, torch.float32, 3, device="cuda"))
    vb, v = _matrix(V, D, torch.float32, 5, 3, wl.normal((V, D), 0.1, torch.float32, 4, device="cuda").square())
    m0, v0 = m.clone(), v.clone()
    opt.embedding_grad_fold(ids, dy, m, v, scale=2.5)
    wm, wv = m0.double() + a * G, v0.double() + b * G * G
    assert bool(((m.double() - wm).abs() <= a * e + U * (wm.abs() + a * e)).all())
    ev = b * (2 * G.abs() + e) * e
    assert bool(((v.double() - wv).abs() <= ev + 3 * U * (wv + ev)).all())
    assert torch.equal(m[~seen], m0[~seen]) and torch.equal(v[~seen], v0[~seen])
    _outside_untouched(mb, m)
    _outside_untouched(vb, v)


@pytest.mark.parametrize("T,V", [(5120, 50257), (5121, 50257), (8192, 50257), (8193, 50257), (20_000, 300), (70_001, 131_072), (200_000, 511), (9000, 512), (9000, 1), (12_345, 300_000)])
@pytest.mark.parametrize("kind", ["text", "padded", "one", "sorted"])
def test_either_way_of_sorting(T, V, kind):
    """Whole numbers: sums are exact in any order, so a token in a wrong place shows."""
    opt = adama.AdamA()
    D = 16
    dy = wl.small_integers((T, D), 8, torch.float32, T).cuda()
    ids = _ids(T, V, kind, 3)
    G = _sums(ids, dy, V, 1.0)[0]
    grad = torch.full((V, D), SENTINEL, device="cuda")
    opt.embedding_grad(ids, dy, grad)
    assert torch.equal(grad.double(), G)
    opt.sync_status()


def test_sums_do_not_depend_on_the_run():
    opt = adama.AdamA()
    for T in (5000, 30_000):
        dy, ids = wl.normal((T, 300), 1.0, torch.float32, 1, device="cuda").bfloat16(), _ids(T, 2000, "text", 5)
        one, two = torch.empty(2000, 300, device="cuda"), torch.empty(2000, 300, device="cuda")
        opt.embedding_grad(ids, dy, one)
        opt.embedding_grad(ids, dy, two)
        assert torch.equal(one, two)


def test_no_tokens():
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    ids, dy = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, 12, device="cuda")
    grad = torch.full((40, 12), SENTINEL, device="cuda")
    opt.embedding(ids, grad, torch.empty(0, 12, device="cuda"))
    opt.embedding_grad(ids, dy, grad, accumulate=True)
    assert bool((grad == SENTINEL).all())
    opt.embedding_grad_fold(ids, dy, grad, grad.clone())
    assert bool((grad == SENTINEL).all())
    opt.embedding_grad(ids, dy, grad)
    assert bool((grad == 0).all())
    opt.embedding_grad(torch.full((9,), -1, dtype=torch.int64, device="cuda"), torch.ones(9, 12, device="cuda"), grad.fill_(SENTINEL))
    assert bool((grad == 0).all())


@pytest.mark.parametrize("T", [50, 9000])
def test_ids_outside_the_table_are_reported(T):
    opt = adama.AdamA()
    V, D = 30, 40
    table = wl.normal((V, D), 1.0, torch.float32, 1).cuda()
    ids = _ids(T, V, "text", 1)
    ids[7], ids[T - 1], ids[3] = V, 1 << 40, -(1 << 40)
    out = torch.empty(T, D, device="cuda")
    opt.embedding(ids, table, out)
    assert torch.isnan(out[[7, T - 1]]).all() and float(out[3].abs().max()) == 0
    fine = (ids >= 0) & (ids < V)
    assert torch.equal(out[fine], table[ids[fine]])
    with pytest.raises(adama.AdamAError) as e:
        opt.sync_status()
    assert e.value.status == Status.ERR_INVALID_ARG and " id " in str(e.value)
    opt.sync_status()
    dy = wl.small_integers((T, D), 8, torch.float32, 2).cuda()
    dy[~fine] = math.nan                                  # rows without a place are not read
    grad = torch.empty(V, D, device="cuda")
    opt.embedding_grad(ids, dy, grad)
    assert torch.equal(grad.double(), _sums(torch.where(fine, ids, -1), dy, V, 1.0)[0])
    with pytest.raises(adama.AdamAError):
        opt.sync_status()
    opt.sync_status()


def test_gradient_against_differences():
    opt = adama.AdamA()
    T, V, D = 9, 4, 5
    ids, dy = _ids(T, V, "text", 4), wl.normal((T, D), 1.0, torch.float32, 1).cuda()
    grad = torch.empty(V, D, device="cuda")
    opt.embedding_grad(ids, dy, grad, scale=3.0)
    table, r = np.zeros((V, D)), dy.double().cpu().numpy()
    for at in np.ndindex(V, D):
        plus, minus = table.copy(), table.copy()
        plus[at] += 1.0
        minus[at] -= 1.0                                   # linear: differences are exact
        slope = (3.0 * (plus - minus)[ids.cpu().numpy()] * r).sum() / 2
        assert abs(float(grad[at]) - slope) <= 1e-5


def test_refusals():
    opt = adama.AdamA()
    ids, table, out = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(5, 8, device="cuda"), torch.ones(3, 8, device="cuda")

    def refused(kind, call, *args, **kw):
        with pytest.raises(kind) as e:
            call(*args, **kw)
        return e.value

    refused(TypeError, opt.embedding, ids.int(), table, out)
    refused(ValueError, opt.embedding, ids[:2], table, out)
    refused(ValueError, opt.embedding, ids, table, out[:, :7])
    refused(ValueError, opt.embedding, ids, table.t(), torch.ones(3, 5, device="cuda"))
    refused(TypeError, opt.embedding, ids, table.half(), out)
    refused(TypeError, opt.embedding, ids.cpu(), table, out)
    for scale in (math.inf, math.nan, 1e39):
        assert refused(adama.AdamAError, opt.embedding, ids, table, out, scale=scale).status == Status.ERR_INVALID_ARG
        assert refused(adama.AdamAError, opt.embedding_grad, ids, out, table, scale=scale).status == Status.ERR_INVALID_ARG
    assert refused(adama.AdamAError, opt.embedding, ids, torch.empty(0, 8, device="cuda"), out).status == Status.ERR_INVALID_ARG
    refused(ValueError, opt.embedding_grad, ids, out, table[:, :7])
    refused(ValueError, opt.embedding_grad_fold, ids, out, table, torch.ones(5, 9, device="cuda")[:, :8])
    refused(TypeError, opt.embedding_grad_fold, ids, out, table.bfloat16(), table.bfloat16())
    assert refused(adama.AdamAError, opt.embedding_grad_fold, ids, out, table, table.clone()).status == Status.ERR_BAD_STATE
    opt.sync_status()
