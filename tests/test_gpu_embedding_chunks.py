"""Gradients of embeddings of so many tokens that a warp takes chunks of 16 (tokens * tiles of 256 columns >= 224 an SM), in all
forms.  Sums of whole numbers times a power of two are exact in any order as long as they stay below 2^24, so a token in a wrong
place, left out or taken twice shows: what is written or added is the exact sum, rounded once where the table is bf16."""
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama
from test_gpu_embedding import TYPES, U, _ids, _matrix, _outside_untouched

pytestmark = pytest.mark.gpu
# one tile; several, the last one whole, even and ragged; ids in more passes of the sort; few tokens and many columns
SHAPES = [(40_001, 500, 250), (40_000, 3000, 256), (36_007, 90_000, 130), (12_000, 700, 601), (9000, 5003, 1028), (5000, 300, 2048), (4100, 37, 2305)]


def _exact(ids, dy, V, scale):
    """The gradient in 64 bits, and which rows have tokens."""
    live = ids >= 0
    g = torch.zeros(V, dy.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids[live], dy[live].double())
    seen = torch.zeros(V, dtype=torch.bool, device="cuda")
    seen[ids[live]] = True
    return g * scale, seen


def _make(T, V, D, dt, kind, pitch, offset):
    assert T * -(-D // 256) // 16 >= 14 * torch.cuda.get_device_properties(0).multi_processor_count
    _, dy = _matrix(T, D, dt, pitch, offset, wl.small_integers((T, D), 8, torch.float32, T + D).cuda())
    return dy, _ids(T, V, kind, T)


@pytest.mark.parametrize("gt,dt", TYPES)
@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("kind,pitch,offset", [("text", 0, 0), ("padded", 3, 1), ("one", 0, 0), ("sorted", 8, 5), ("even", 1, 0)])
def test_written_and_added(T, V, D, gt, dt, kind, pitch, offset):
    opt = adama.AdamA()
    dy, ids = _make(T, V, D, dt, kind, pitch, offset)
    G, seen = _exact(ids, dy, V, 0.5)
    assert float(G.abs().max()) < 2 ** 24
    buf, grad = _matrix(V, D, gt, pitch, offset)
    opt.embedding_grad(ids, dy, grad, scale=0.5)
    assert torch.equal(grad, G.float().to(gt))
    _outside_untouched(buf, grad)
    start = wl.small_integers((V, D), 8, torch.float32, V).cuda().to(gt)
    grad.copy_(start)
    opt.embedding_grad(ids, dy, grad, scale=0.5, accumulate=True)
    assert torch.equal(grad, (start.double() + G).float().to(gt))
    _outside_untouched(buf, grad)
    opt.sync_status()


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("kind,pitch,offset", [("text", 0, 0), ("padded", 5, 3), ("one", 0, 0), ("sorted", 4, 0), ("even", 1, 0)])
def test_folded(T, V, D, dt, kind, pitch, offset):
    """The sum is exact; a fold rounds m once (u of the result), v at most three times."""
    opt = adama.AdamA()
    opt.begin_minibatch(4)
    a, b = (float(c) for c in adama.host_constants(0.9, 0.999, 1e-8, 4, 1, 1e-3)[:2])
    dy, ids = _make(T, V, D, dt, kind, 0 if pitch == 0 else 8, offset)
    G, seen = _exact(ids, dy, V, 2.0)
    mb, m = _matrix(V, D, torch.float32, pitch, offset, wl.normal((V, D), 0.1, torch.float32, 3, device="cuda"))
    vb, v = _matrix(V, D, torch.float32, pitch, offset, wl.normal((V, D), 0.1, torch.float32, 4, device="cuda").square())
    m0, v0 = m.clone(), v.clone()
    opt.embedding_grad_fold(ids, dy, m, v, scale=2.0)
    wm, wv = m0.double() + a * G, v0.double() + b * G * G
    assert bool(((m.double() - wm).abs() <= U * wm.abs()).all())
    assert bool(((v.double() - wv).abs() <= 3 * U * wv).all())
    assert torch.equal(m[~seen], m0[~seen]) and torch.equal(v[~seen], v0[~seen])
    _outside_untouched(mb, m)
    _outside_untouched(vb, v)
    opt.sync_status()
