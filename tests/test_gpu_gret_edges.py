"""Gated retention where its kernels meet their borders."""
import time

import numpy as np
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


@pytest.mark.parametrize("lens", [[1, 1, 1], [40, 300, 17]], ids=str)
def test_an_output_over_an_input_is_refused_and_one_beside_them_is_not(lens):
    """Nothing is enqueued by the refused calls: states and rows stay."""
    import torch
    H, d, step = 2, 64, max(lens) == 1
    p = Problem(lens, H, d, seed=107, norm="rms", in_place=True)
    yx, n, W = p.yx, sum(lens), H * d
    x = torch.zeros(n + 8, 5 * W + 16, dtype=torch.bfloat16, device="cuda")
    for i, t in enumerate((p.q, p.k, p.v, p.gate)):
        x[:n, i * W:(i + 1) * W] = t
    S, flat = x.shape[1], x.view(-1)
    col = lambda i, row=0: x[row:row + n, i * W:(i + 1) * W]  # noqa: E731
    ng = yx.make_norm_gate(1e-5, rms=True, gate=col(3), gate_stride=S)

    def call(o, o_stride, q=None, q_stride=S, decay=p.decay, ng=ng):
        shape = yx.make_gret_shape(len(lens), H, d, num_slots=p.n_slots, tau=p.tau, q_stride=q_stride, k_stride=S, v_stride=S, o_stride=o_stride)
        rows = (col(0) if q is None else q, col(1), col(2), decay, ng, p.state, p.slot_in, p.slot_out)
        if step:
            yx.yoco_gret_step(shape, *rows, o)
        else:
            ws = torch.empty(yx.yoco_gret_workspace_size(shape, lens), dtype=torch.uint8, device="cuda")
            yx.yoco_gret_chunk(shape, *rows, lens, o, ws)

    before = x.clone()
    dense = flat[8:8 + n * W].view(n, W)                     # over columns of everything
    gap = flat[16:16 + n * (W + 8)].view(n, W + 8)[:, :W]    # starts inside Q's first row
    over = [(col(i), S) for i in range(4)] + [(col(i, 1), S) for i in range(4)] + [(x[:n, W // 2:W // 2 + W], S), (x[:n, 3 * W + 8:4 * W + 8], S), (dense, W), (gap, W + 8)]
    bytes_of = torch.zeros(4 * n * W, dtype=torch.uint8, device="cuda")
    shared = bytes_of[:2 * n * W].view(torch.bfloat16).view(n, W)
    for o, stride in over:
        with pytest.raises(yx.YocoError) as e:
            call(o, stride)
        assert e.value.code == yx.ERR_INVALID_ARG, (o.storage_offset(), stride)
    with pytest.raises(yx.YocoError):
        call(shared, W, decay=bytes_of.view(torch.float32)[:n * H].view(n, H))
    with pytest.raises(yx.YocoError):
        call(shared, W, q=shared, q_stride=W)
    torch.cuda.synchronize()
    assert torch.equal(x, before) and np.array_equal(p.state.cpu().numpy(), p.state0)
    # beside them: the fifth part of the same buffer
    p.norm, p.shape.o_stride = None, S
    o = col(4)
    o.fill_(0)
    call(o, S, ng=None)
    assert torch.equal(x[:n, :4 * W], before[:n, :4 * W]) and torch.equal(x[n:], before[n:]) and bool((x[:, 5 * W:] == 0).all())
    p.o_buf[1:n + 1, :W] = o
    p.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,H", [([300, 40, 129], 60), ([2600, 777], 3)], ids=["whole", "cut"])
def test_an_expired_wait_is_reported_and_the_next_call_is_correct(lens, H, d):
    """A producer that starts no copy: every role of the kernel gives up its first wait, with nothing in flight, the CTAs leave in the ordinary way, the
    host reads which wait it was, and the next call on the same workspace and states is right."""
    import torch
    p = Problem(lens, H, d, seed=109, norm="group")
    yx = p.yx
    ws = torch.zeros(p.workspace()[1], dtype=torch.uint8, device="cuda")
    assert (ws.numel() > 0) == (H == 3)
    assert yx.yoco_kv_append_status() == 0
    t0 = time.perf_counter()
    yx.yoco_gret_selftest_wait_expiry(p.shape, p.q, p.k, p.v, p.decay, p.ng, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws, limit_ms=20)
    rc, wait_class, cta = yx.yoco_kv_append_status_detail()
    dt = time.perf_counter() - t0
    assert rc == yx.ERR_TIMEOUT and wait_class in (yx.WAIT_RING_FULL, yx.WAIT_TENSOR) and 0 <= cta < 148
    assert 0.015 < dt < 2.0, dt                               # the limit was honoured, once per kernel
    assert yx.yoco_kv_append_status() == 0                    # cleared
    p.state.copy_(torch.from_numpy(p.state0))
    yx.yoco_gret_chunk(p.shape, p.q, p.k, p.v, p.decay, p.ng, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
    assert yx.yoco_kv_append_status() == 0
    p.check()
    short = yx.make_gret_shape(len(lens), H, d, T=5, num_slots=p.n_slots, tau=p.tau, q_stride=4 * H * d, k_stride=4 * H * d, v_stride=4 * H * d)
    with pytest.raises(yx.YocoError) as e:                    # token by token: no waits
        yx.yoco_gret_selftest_wait_expiry(short, p.q, p.k, p.v, p.decay, None, p.state, p.slot_in, p.slot_out, None, torch.empty_like(p.o), ws, limit_ms=20)
    assert e.value.code == yx.ERR_UNSUPPORTED
