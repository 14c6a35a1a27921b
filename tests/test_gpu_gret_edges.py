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


def test_one_workspace_while_sequences_leave_a_batch():
    import torch
    H, d, lens = 32, 64, [900] * 8
    p = Problem(lens, H, d, seed=103, in_place=True)
    ws = torch.empty(p.yx.yoco_gret_workspace_bound(p.shape, lens), dtype=torch.uint8, device="cuda")
    for left in (8, 1):
        q = Problem(lens[:left] + [0] * (8 - left), H, d, seed=104 + left, in_place=True)
        q.yx.yoco_gret_chunk(q.shape, q.q, q.k, q.v, q.decay, None, q.state, q.slot_in, q.slot_out, q.lens, q.o, ws)
        q.check()
    assert p.yx.yoco_gret_workspace_size(p.shape, lens) < p.yx.yoco_gret_workspace_size(q.shape, q.lens) <= ws.numel()
    assert p.yx.yoco_kv_append_status() == 0
