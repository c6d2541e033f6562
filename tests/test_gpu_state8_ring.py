"""Lists of 8-bit states that are long enough to be streamed, made of what the bulk copies do not
bring: ragged last blocks, tensors shorter than a chunk, tensors without alignment."""
import pytest
import torch

import paper_2305_19982_b200 as adama
from paper_2305_19982_b200 import State8, State8List

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offset", [0, 1])
def test_ragged_tensors_of_a_streamed_list_equal_one_at_a_time(offset):
    """447 tensors of up to 2.5 chunks (4096 elements): nearly every chunk has warps whose block is
    ragged, or that have none.  Same bits as calls of one tensor each, which take no ring."""
    gen = torch.Generator(device="cuda").manual_seed(offset)
    sizes = [1 + (2657 * i) % 10_007 for i in range(447)]
    make = lambda dtype, std: [(torch.randn(n + 1, generator=gen, device="cuda") * std).to(dtype)[offset:offset + n] for n in sizes]  # noqa: E731
    ws, gs = make(torch.float32, 0.02), make(torch.bfloat16, 1e-3)
    w2 = [w.clone() for w in ws]
    one, many = [State8.zeros(n) for n in sizes], [State8.zeros(n) for n in sizes]
    a, b = adama.AdamA(), adama.AdamA()
    for _ in range(3):
        a.begin_minibatch(1)
        b.begin_minibatch(1)
        a.fold_apply8_multi(ws, gs, State8List(many), 1e-3)
        for w, g, s in zip(w2, gs, one):
            b.fold_apply8_multi([w], [g], [s], 1e-3)
    a.sync_status()
    b.sync_status()
    assert a.launch_count == 3
    for x, y, s, t in zip(ws, w2, many, one):
        assert torch.equal(x, y) and torch.equal(s.v_codes, t.v_codes)
        assert torch.equal(s.m_codes.view(torch.uint8), t.m_codes.view(torch.uint8))
        assert torch.equal(s.m_scale, t.m_scale) and torch.equal(s.v_scale, t.v_scale)
