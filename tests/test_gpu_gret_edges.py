"""Gated retention where its kernels meet their borders."""
import pytest

from test_gpu_gret import Problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_state_only_ranges_that_end_one_stream_and_begin_another(d):
    """Every third CTA's range has the end of one stream and the beginning of the next: the makers of K' go from segment to segment, each at its own
    pace.  The same call over and over gives the same bits, and no wait runs out."""
    import torch
    p = Problem([1500, 1409, 1530], 16, d, seed=101)         # 48 streams of 12 chunks, 576 chunks over the CTAs
    ws, n = p.workspace()
    assert n > 0
    p.chunk().check()
    o, state = p.o.clone(), p.state.clone()
    call = p.yx.prepare_tokens("yoco_gret_chunk", p.shape, p.q, p.k, p.v, p.decay, None, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
    for _ in range(40):
        p.o.zero_()
        call.run()
        assert torch.equal(p.o, o) and torch.equal(p.state, state)
    assert p.yx.yoco_kv_append_status() == 0
