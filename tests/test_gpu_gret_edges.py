"""Gated retention where its kernels meet their borders."""
import functools
import time

import numpy as np
import pytest

import gret_ref
from test_gpu_gret import GUARD, Problem

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


# ---- row by row -----------------------------------------------------------------------------------------
# In chunks of 128 tokens the scores with their decays (P) and the copy of the state that meets Q are rounded to bf16, each element by up to 2^-8 of its value,
# independently of the others.  An output is a sum of such elements times exact numbers, so its error is above 7 * 2^-8 * sqrt(sum of the terms'
# squares) with a probability of at most 2 exp(-7^2 / 2) = 5e-11 (Hoeffding).  Beside that come operations in fp32 and the second part of the weights inside cut
# streams, 2^-16 of the sum of magnitudes, and the output's own rounding.
U = 2.0 ** -8


def squares(p):
    """sqrt of the sums of the squares of an output's terms, [tokens, H, d]."""
    H, d = p.H, p.d
    f = lambda t: t.double().cpu().numpy().reshape(-1, H, d).transpose(1, 0, 2)  # noqa: E731
    q, k, v = f(p.q) * (p.scale or d ** -0.5), f(p.k), f(p.v)
    logs = np.maximum(gret_ref.log_decay(p.decay.float().cpu().numpy(), p.tau), -110.0).T
    out, first = np.zeros_like(q), 0
    for n, slot in zip(p.lens, p.slot_in):
        s = np.zeros((H, d, d)) if slot < 0 else p.state0[slot].astype(np.float64)
        for c in range(first, first + n, 128):
            at = slice(c, min(c + 128, first + n))
            b = logs[:, at].cumsum(1)
            e = np.exp(np.minimum(b[:, :, None] - b[:, None], 0.0)) * np.tri(b.shape[1])
            P, qs = (q[:, at] @ k[:, at].transpose(0, 2, 1)) * e, q[:, at] * np.exp(b)[:, :, None]
            out[:, at] = np.sqrt(P ** 2 @ v[:, at] ** 2 + qs ** 2 @ s ** 2)
            s = np.exp(b[:, -1])[:, None, None] * s + (k[:, at] * np.exp(b[:, -1:] - b)[:, :, None]).transpose(0, 2, 1) @ v[:, at]
        first += n
    return out.transpose(1, 0, 2)


def check_rows(p, in_chunks=True):
    """Every element of the output (its norm's bound follows from the bounds of the row's elements), then states and surroundings."""
    n, H, d = sum(p.lens), p.H, p.d
    o, o_abs, _, _ = p.reference()
    spread = squares(p) if in_chunks else np.zeros_like(o)
    t = 7 * U * spread + 2.0 ** -16 * o_abs
    f = lambda x, *s: None if x is None else x.double().cpu().numpy().reshape(*s)  # noqa: E731
    got = f(p.o, n, H, d)
    if p.norm is None:
        want, tol, size = o, t, spread
    else:
        rms, gate, gain, bias = p.norm == "rms", f(p.gate, n, H, d), f(p.gain, H, d), f(p.bias, H, d)
        want = gret_ref.norm_gate(o, 1e-5, rms, gate, gain, bias)
        swish = np.abs(gate / (1 + np.exp(-gate)))
        factor = swish * (1.0 if gain is None else np.abs(gain))
        x = np.abs(gret_ref.norm_gate(o, 1e-5, rms))
        root = np.sqrt((o * o).mean(-1, keepdims=True) + 1e-5) if rms else np.sqrt(o.var(-1, keepdims=True) + 1e-5)
        off = np.sqrt((t * t).mean(-1, keepdims=True))      # how far the root may be off
        assert (off < root).all(), "the norm leaves nothing to compare"
        tol = factor * (t + (0.0 if rms else t.mean(-1, keepdims=True)) + x * off) / (root - off)
        tol = tol + 2.0 ** -18 * (factor * (1 + x) + swish)  # sums of d values, root, exponential, reciprocal
        size = factor * spread / root
    tol = tol + U * np.abs(want) + 1e-30
    worst = np.abs(got - want) / tol
    assert np.isfinite(got).all() and worst.max() <= 1, (np.unravel_index(worst.argmax(), worst.shape), worst.max())
    # all together: uniformly distributed errors have a third of the square of the largest one on average
    together = np.linalg.norm(got - want) / np.sqrt(((U * want) ** 2 + (U * size) ** 2).sum() / 3)
    assert together <= 1.5, together
    p.norm, norm = None, p.norm
    if norm is None:
        p.check()
    else:
        rows = p.o.clone()
        p.o.copy_(torch_bf16(o, p.o))                       # (the norm's output has been looked at: states and surroundings)
        p.check()
        p.o.copy_(rows)
    p.norm = norm
    return np.linalg.norm(got - want) / np.linalg.norm(want)


def torch_bf16(x, like):
    import torch
    return torch.from_numpy(x.reshape(like.shape)).to(torch.bfloat16).to(like.device)


@functools.lru_cache(None)
def longest_walked(B, H, d):
    """The longest length up to which calls of B sequences are walked token by token (the self-test of the chunkwise kernel's waits refuses those)."""
    import torch
    p = Problem([64] * B, H, d, seed=1)
    for n in range(1, 65):
        shape = p.yx.make_gret_shape(B, H, d, T=n, num_slots=p.n_slots, tau=p.tau, q_stride=4 * H * d, k_stride=4 * H * d, v_stride=4 * H * d, o_stride=H * d + GUARD)
        ws = torch.empty(p.yx.yoco_gret_workspace_size(shape), dtype=torch.uint8, device="cuda")
        try:
            p.yx.yoco_gret_selftest_wait_expiry(shape, p.q, p.k, p.v, p.decay, None, p.state, p.slot_in, p.slot_out, None, p.o, ws, limit_ms=1)
        except p.yx.YocoError as e:
            assert e.code == p.yx.ERR_UNSUPPORTED
            continue
        assert p.yx.yoco_kv_append_status() == p.yx.ERR_TIMEOUT
        return n - 1
    return 64


def walked_lengths(H, d):
    """Lengths that are walked token by token: the longest, and ends before, on and behind a batch of eight tokens."""
    for lens in ([0], [5, 0], [8, 9, -1], [1, 0, 0], [7, 16, 0]):
        n = longest_walked(len(lens), H, d)
        yield [min(x, n) if x > 0 else n + x for x in lens]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(), dict(norm="group"), dict(norm="rms", gain=True, bias=True), dict(norm="group", gain=True, bias=True, in_place=True),
                                dict(tau=0.0, fresh=(0,)), dict(tau=16.0, scale=0.7)], ids=str)
def test_rows_of_tokens_walked_one_by_one(kw, d):
    for i, lens in enumerate(walked_lengths(3, d)):
        p = Problem(lens, 3, d, seed=120 + i, **kw).chunk()
        check_rows(p, in_chunks=False)
    n = longest_walked(1, 3, d)                              # on the other side of the border
    check_rows(Problem([n + 1], 3, d, seed=130, **kw).chunk())


@pytest.mark.parametrize("d", [64, 128])
def test_strong_decays_of_tokens_walked_one_by_one(d):
    r = np.random.RandomState(6)
    H = 2
    for i, lens in enumerate(walked_lengths(H, d)):
        n = sum(lens)
        logs = -0.002 * r.rand(n, H)
        logs[r.rand(n) < 0.2] = -100.0
        logs[r.rand(n) < 0.1] = -1e4
        logs[r.rand(n) < 0.1] = -np.inf
        logs[n // 2] = -60.0
        check_rows(Problem(lens, H, d, tau=0.0, logs=logs, seed=140 + i).chunk(), in_chunks=False)
        z = np.where(r.rand(n, H) < 0.2, -3e4, 30.0)
        check_rows(Problem(lens, H, d, tau=16.0, logs=z, seed=150 + i, norm="rms").chunk(), in_chunks=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(), dict(norm="group"), dict(norm="rms", gain=True, bias=True), dict(norm="group", gain=True, bias=True)], ids=str)
def test_rows_of_chunks(kw, d):
    """Streams whole, cut, and several to a range."""
    for i, (lens, H) in enumerate((([300, 26, 140, 129] * 10, 4), ([700, 256], 2), ([1900, 3, 777, 1300], 6))):
        check_rows(Problem(lens, H, d, seed=160 + i, **kw).chunk())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("offset", [3.0, 10.0])
def test_a_norm_that_takes_a_common_offset_out(offset, d):
    """Values around an offset: the norm takes out what most of P's and the state's roundings were relative to."""
    for lens, H in (([300, 140], 40), ([384], 3)):
        p = Problem(lens, H, d, seed=170, norm="group", fresh=range(len(lens)))
        p.v += offset
        print("offset", offset, lens, d, check_rows(p.chunk()))
