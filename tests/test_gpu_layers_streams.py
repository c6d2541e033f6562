"""Norms, embeddings and the distillation loss among other work: several streams, graphs that are played in another order
than they were recorded in, workspaces that grow, rows further apart than 32-bit offsets reach."""
import pytest
import torch

import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import Status

pytestmark = pytest.mark.gpu


def _rand(shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to("cuda", dtype)


def _work(opt, rows, dim, vocab, seed):
    """One call of each kind, as (call, outputs), and what they gave when each ran alone on the default stream."""
    x, dy, w, b = (_rand(s, seed + i, t) for i, (s, t) in enumerate([((rows, dim), torch.bfloat16), ((rows, dim), torch.bfloat16),
                                                                    ((dim,), torch.float32), ((dim,), torch.float32)]))
    table = _rand((vocab, dim), seed + 5, torch.bfloat16)
    g = torch.Generator().manual_seed(seed + 6)
    ids = (torch.rand(rows, generator=g) ** 3 * vocab).long().cuda()
    logits, teacher = _rand((rows, vocab), seed + 7, torch.bfloat16), _rand((rows, 5), seed + 8)
    entries, weights = torch.randint(0, vocab, (rows, 5), generator=g).cuda(), torch.rand(rows, generator=g).cuda()
    y, dx, e, dl = (torch.empty_like(t) for t in (x, x, x, logits))
    mean, rstd = torch.empty(2, rows, device="cuda")
    dw, db, stats, grad = (torch.empty(s, device="cuda") for s in ((dim,), (dim,), (4,), (vocab, dim)))
    calls = [
        (lambda: opt.embedding(ids, table, e, 0.5), [e]),
        (lambda: opt.layer_norm(x, w, b, y, mean, rstd), [y, mean, rstd]),
        (lambda: opt.distill_loss(logits, teacher, entries, weights, dl, stats), [dl, stats]),
        (lambda: opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db), [dx, dw, db]),
        (lambda: opt.embedding_grad(ids, dy, grad), [grad]),
    ]
    out = [t for _, outs in calls for t in outs]
    for call, _ in calls:
        call()
        torch.cuda.synchronize()
    want = [t.clone() for t in out]
    return [c for c, _ in calls], out, want


def _spoil(works):
    for _, out, _ in works:
        for t in out:
            t.fill_(-1.0)
    torch.cuda.synchronize()


def _check(works):
    torch.cuda.synchronize()
    for _, out, want in works:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


SIZES = [(700, 160, 301), (9000, 96, 613), (33, 1600, 5003), (1, 1, 2)]


def test_calls_on_several_streams_at_once():
    opt = adama.AdamA()
    works = [_work(opt, *s, seed=i) for i, s in enumerate(SIZES)]
    streams = [torch.cuda.Stream() for _ in works]
    for turn in range(20):
        _spoil(works)
        for (calls, _, _), s in zip(works[turn % 2:] + works[:turn % 2], streams):
            with torch.cuda.stream(s):
                for _ in range(3):
                    for c in calls:
                        c()
        _check(works)
    opt.sync_status()


def test_graphs_in_any_order_and_between_other_calls():
    """Recorded on one stream, whose eager calls' workspace grows in between; played at once on several."""
    opt = adama.AdamA()
    works = [_work(opt, *s, seed=10 + i) for i, s in enumerate(SIZES)]
    side = torch.cuda.Stream()
    graphs = []
    for i, (calls, _, _) in enumerate(works[:3]):
        if i == 1:
            with torch.cuda.stream(side):
                for c in works[3][0]:
                    c()
            side.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            for c in calls:
                c()
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        _spoil(works)
        for g, s in list(zip(graphs, streams))[::-1]:
            with torch.cuda.stream(s):
                for _ in range(3):
                    g.replay()
        with torch.cuda.stream(side):
            for c in works[3][0]:
                c()
        _check(works)
    opt.sync_status()


def test_one_workspace_for_calls_of_all_sizes():
    opt = adama.AdamA()
    works = [_work(opt, *s, seed=20 + i) for i, s in enumerate([(3, 24, 50), (20_000, 8, 700), (5, 9000, 40), (300, 300, 300)])]
    _spoil(works)
    with torch.cuda.stream(torch.cuda.Stream()):
        for calls in zip(*[w[0] for w in works]):
            for c in calls:
                c()
    _check(works)


@pytest.mark.parametrize("dim", [40, 1601])
def test_offsets_past_32_bits(dim):
    """Three rows, 2^30 elements apart: what the same rows give close together."""
    opt = adama.AdamA()
    ld, rows = 1 << 30, 3
    big = torch.empty(2 * ld + dim, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((rows, dim), (ld, 1))
    x, dy, w = _rand((rows, dim), 1, torch.bfloat16), _rand((rows, dim), 2, torch.bfloat16), _rand((dim,), 3)
    ids = torch.tensor([2, 0, 2], device="cuda")

    def both(call):
        """call(matrix): through the far rows, which hold x before, and through near ones, which start as aligned."""
        near = torch.empty(rows, -(-dim // 64) * 64, dtype=torch.bfloat16, device="cuda")[:, :dim]
        near.copy_(x)
        far.copy_(x)
        first, second = call(far), call(near)
        assert torch.equal(far, near)
        assert all(torch.equal(a, b) for a, b in zip(first, second))

    def norm(t):
        mean, rstd = torch.empty(2, rows, device="cuda")
        opt.layer_norm(t, w, None, t, mean, rstd)
        return [mean, rstd]

    def norm_back(t):
        mean, rstd, dw = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda"), torch.empty(dim, device="cuda")
        opt.layer_norm_backward(dy, t, w, mean, rstd, t, dw)
        return [dw]

    def lookup(t):
        e = torch.empty(rows, dim, device="cuda")
        opt.embedding(ids, t, e)
        return [e]

    def distill(t):
        stats, loss = torch.empty(4, device="cuda"), torch.empty(rows, device="cuda")
        opt.distill_loss(t, dy[:, :4], torch.tensor([[1, 5, 9, 2]] * rows, device="cuda"), w[:rows].abs(), t, stats, loss=loss)
        return [stats, loss]

    def table_grad(t):
        opt.embedding_grad(ids, dy, t, accumulate=True)
        return []

    for call in (norm, norm_back, lookup, distill, table_grad):
        both(call)
    far.fill_(7.0)
    grad = torch.full((rows, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    opt.embedding_grad(ids, dy, far)
    opt.embedding_grad(ids, dy, grad)
    assert torch.equal(far, grad) and not bool(grad[1].any())
    opt.sync_status()


def test_rows_of_the_gradient_are_refused_from_a_length_on():
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    wide = torch.zeros(1, (1 << 23) + 1, device="cuda")
    ids = torch.zeros(1, dtype=torch.int64, device="cuda")
    for call in (lambda: opt.embedding_grad(ids, wide, wide.clone()), lambda: opt.embedding_grad_fold(ids, wide, wide.clone(), wide.clone())):
        with pytest.raises(adama.AdamAError) as e:
            call()
        assert e.value.status == Status.ERR_UNSUPPORTED
    grad = torch.full((2, 1 << 23), 3.0, device="cuda")
    opt.embedding_grad(ids, wide[:, 1:] + 1.5, grad)        # the longest row
    assert bool((grad[0] == 1.5).all()) and not bool(grad[1].any())
    out = torch.empty(1, wide.shape[1], device="cuda")
    opt.embedding(ids, wide + 2.5, out)
    assert bool((out == 2.5).all())
    opt.sync_status()


@pytest.mark.parametrize("T", [1, 50, 9000])
@pytest.mark.parametrize("D", [5, 64, 1028])
def test_a_batch_of_nothing_but_padding(T, D):
    opt = adama.AdamA()
    opt.begin_minibatch(1)
    ids = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    dy, table = torch.full((T, D), float("nan"), device="cuda"), torch.full((77, D), 3.0, device="cuda")
    out = torch.full((T, D), 7.0, device="cuda")
    opt.embedding(ids, table, out)
    assert not bool(out.any())
    m, v, grad = (torch.full((77, D), 3.0, device="cuda") for _ in range(3))
    opt.embedding_grad_fold(ids, dy, m, v)
    opt.embedding_grad(ids, dy, grad, accumulate=True)
    assert all(torch.equal(t, table) for t in (m, v, grad))
    opt.embedding_grad(ids, dy, grad)
    assert not bool(grad.any())
    # a distillation of which no row counts
    logits, d = torch.full((T, 3 * D), float("nan"), device="cuda"), torch.full((T, 3 * D), 7.0, device="cuda")
    stats, loss = torch.full((4,), 7.0, device="cuda"), torch.full((T,), 7.0, device="cuda")
    opt.distill_loss(logits, dy[:, :5], ids[:, None].expand(T, 5).contiguous(), torch.zeros(T, device="cuda"), d, stats, loss=loss)
    assert not bool(d.any()) and not bool(stats.any()) and not bool(loss.any())
    opt.sync_status()


def test_calls_from_several_threads():
    """A context and a stream to each thread, the same inputs."""
    import threading
    x, w, ids, dy = _rand((500, 1600), 1), _rand((1600,), 2), (torch.arange(500) % 37).cuda(), _rand((500, 1600), 3)
    results, errors = [], []

    def work():
        try:
            opt, y, grad = adama.AdamA(), torch.empty_like(x), torch.empty(37, 1600, device="cuda")
            mean, rstd = torch.empty(2, 500, device="cuda")
            dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(50):
                    opt.layer_norm(x, w, None, y, mean, rstd)
                    opt.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
                    opt.embedding_grad(ids, dy, grad)
                torch.cuda.current_stream().synchronize()
            opt.sync_status()
            results.append((y, dx, dw, db, grad))
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    assert all(torch.equal(a, b) for r in results[1:] for a, b in zip(r, results[0]))
