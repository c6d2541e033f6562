"""The reductions' scratch under CUDA-graph capture: a graph carries the zero-fill of the scratch that
its calls use, and shares that scratch with nothing else."""
import pytest
import torch

import adama_workloads as wl
import paper_2305_19982_b200 as adama

pytestmark = pytest.mark.gpu


def _spoil(pool):
    """Leaves memory of the pool filled, so that scratch taken from it is not zero by luck."""
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, pool=pool):
        blocks = [torch.full((65536,), 0x40, dtype=torch.uint8, device="cuda") for _ in range(16)]
        del blocks
    g.replay()
    torch.cuda.synchronize()
    return g


def _norm_calls(opt):
    """A norm over several thread blocks: (call, output, what it should be)."""
    x = wl.normal((300_000,), 1e-2, torch.float32, 3).cuda()
    out, want = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    adama.AdamA().grad_norm_multi([x], 0.5, want)
    lists = adama.TensorList([x])
    return (lambda: opt.grad_norm_multi(lists, 0.5, out)), out, want


def _policy_calls(opt):
    """A loss over several thread blocks: (call, stats, what they should be)."""
    T, V = 600, 1031
    x = wl.normal((T, V), 2.0, torch.float32, 5).cuda()
    targets = torch.arange(T, device="cuda")
    logp, d = torch.empty(T, device="cuda"), torch.empty(T, V, device="cuda")
    out, want = torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    ref = adama.AdamA()
    ref.token_logprobs(x, targets, logp)
    one = torch.ones(T, device="cuda")
    ref.policy_loss(x, targets, logp - 0.1, one, one, d, want, ref_logp=logp - 0.3, kl_coef=0.1)
    old, other = logp - 0.1, logp - 0.3
    return (lambda: opt.policy_loss(x, targets, old, one, one, d, out, ref_logp=other, kl_coef=0.1)), out, want


CALLS = [_norm_calls, _policy_calls]


@pytest.mark.parametrize("calls", CALLS)
@pytest.mark.parametrize("first_played", [False, True])
def test_two_graphs_of_one_stream_played_in_reverse(calls, first_played):
    """The context's first calls are recorded, not run; the graph recorded second is played first, or alone."""
    opt = adama.AdamA()
    call, out, want = calls(opt)
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    keep = _spoil(pool)                                      # noqa: F841 - owns the pool's memory
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g in graphs:
        with torch.cuda.graph(g, pool=pool):
            call()
            call()
    for g in reversed(graphs) if first_played else graphs[1:]:
        out.fill_(-1.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    out.fill_(-1.0)
    call()                                                    # not recorded
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("calls", CALLS)
def test_graphs_played_on_several_streams_and_calls_beside_them(calls):
    """Three graphs recorded on one stream, one of them after a plain call on it, played on streams of their
    own while plain calls go on: every result is right every time."""
    opt = adama.AdamA()
    record = torch.cuda.Stream()
    made = [calls(opt) for _ in range(4)]
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in range(3)]
    for i, (call, _, _) in enumerate(made[:3]):
        if i == 1:
            with torch.cuda.stream(record):
                call()
            record.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=record):
            call()
        graphs.append(g)
    for _ in range(20):
        for _, out, _ in made:
            out.fill_(-1.0)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                for _ in range(5):
                    g.replay()
        with torch.cuda.stream(record):
            for _ in range(5):
                made[3][0]()
        torch.cuda.synchronize()
        for _, out, want in made:
            assert torch.equal(out, want)


def test_a_clipped_update_in_a_graph():
    """Norm, factor and update recorded together: what the plain calls give."""
    n = 200_001
    res = []
    for recorded in (False, True):
        opt = adama.AdamA()
        w, g = wl.normal((n,), 0.02, torch.float32, 1).cuda(), wl.normal((n,), 1e-2, torch.bfloat16, 2).cuda()
        m, v, out = torch.zeros_like(w), torch.zeros_like(w), torch.empty(4, device="cuda")
        lists = [adama.TensorList([t]) for t in (w, g, m, v)]
        opt.begin_minibatch(1)

        def step():
            opt.grad_norm_multi(lists[1], 0.5, out)
            opt.fold_apply_multi(*lists, 1e-3, grad_factor=out[1:2])

        if recorded:
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            graph.replay()
        else:
            step()
        torch.cuda.synchronize()
        res.append((w, m, v, out))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_capture_ids_tell_graphs_apart():
    L, stream, ids = adama.load_library(), torch.cuda.Stream(), []
    for _ in range(2):
        assert L.adama_stream_capture_id(stream.cuda_stream) == 0
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=stream):
            ids.append(L.adama_stream_capture_id(stream.cuda_stream))
            assert L.adama_stream_capture_id(torch.cuda.default_stream().cuda_stream) == 0
            torch.zeros(8, device="cuda")
    assert 0 not in ids and ids[0] != ids[1]
