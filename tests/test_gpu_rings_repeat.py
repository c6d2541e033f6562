"""Kernels that stream through a ring in shared memory, run many times on the same inputs: a stage that were filled anew while it
is still read would show as a result that differs, in few runs of many."""
import pytest
import torch

import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import State8, State8List, TensorList

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# rings of 64, 128, 256, 512 and 640 threads, and a cluster's; logits and gradient in step, or shifted against each other
@pytest.mark.parametrize("T,V", [(3000, 4096), (2000, 6000), (2000, 12_000), (1200, 24_000), (800, 32_768), (500, 60_000), (400, 120_000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("pitch", [0, 2])
def test_policy_loss(T, V, dtype, pitch):
    opt, gen = adama.AdamA(), _gen(T + V)
    x = torch.randn(T, V, generator=gen, device="cuda").mul_(2).to(dtype)
    targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
    old, adv, weights = (torch.rand(T, generator=gen, device="cuda") for _ in range(3))
    old = -3 * old
    weights[::4] = 0.0
    d = torch.empty(T, V + pitch, dtype=torch.bfloat16, device="cuda")[:, :V]
    stats, logp = torch.empty(4, device="cuda"), torch.empty(T, device="cuda")
    first, differ = None, torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        opt.policy_loss(x, targets, old, adv, weights, d, stats, logp=logp)
        if first is None:
            first = [r.clone() for r in (d, stats, logp)]
        differ += sum((a != b).any() for a, b in zip((d, stats, logp), first))
    assert int(differ) == 0
    opt.sync_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_updates(dtype, bits):
    """From the same weights and moments every time: ten tensors, one of them with a ragged end."""
    opt, gen = adama.AdamA(), _gen(bits)
    sizes = [2_560_000] * 5 + [1600] * 4 + [999_424 + 77]
    opt.begin_minibatch(1)
    start = [torch.randn(n, generator=gen, device="cuda").mul_(0.02) for n in sizes]
    w, copy = [t.clone() for t in start], [torch.empty_like(t, dtype=torch.bfloat16) for t in start]
    grads = TensorList([torch.randn(n, generator=gen, device="cuda").mul_(1e-3).to(dtype) for n in sizes])
    if bits == 8:
        states = [State8.zeros(n) for n in sizes]
        parts = [t for s in states for t in (s.m_codes.view(torch.uint8), s.m_scale, s.v_codes, s.v_scale)]
        opt.fold_apply8_multi(TensorList(w), grads, State8List(states), 1e-3)       # moments that are not zero
        lists = (State8List(states),)
        call = opt.fold_apply8_multi
    else:
        moments = [[torch.randn(n, generator=gen, device="cuda").mul_(1e-3) for n in sizes] for _ in range(2)]
        for t in moments[1]:
            t.square_()
        parts = moments[0] + moments[1]
        lists = tuple(TensorList(t) for t in moments)
        call = opt.fold_apply_multi
    saved, weights, copies = [t.clone() for t in parts], TensorList(w), TensorList(copy)
    first, differ = None, torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        for t, s in zip(w + parts, start + saved):
            t.copy_(s)
        opt.set_step(1)
        opt.begin_minibatch(1)
        call(weights, grads, *lists, 1e-3, w_bf16=copies)
        if first is None:
            first = [t.clone() for t in w + copy + parts]
        differ += sum((a != b).any() for a, b in zip(w + copy + parts, first))
    assert int(differ) == 0
    opt.sync_status()
