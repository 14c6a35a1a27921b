"""Head norm with gate and rotation of token-major rows on the GPU against 64 bits, and a self-decoder's attention-like module as it is used:
rotation, retention with norm and gate, prompt then single tokens.

A result that is rounded to bf16 once is off by at most 2^-8 of its value; before that come fp32 operations: for the rotation three
(2^-24 each, relative to |x1| + |x2|) and cosines and sines to 2^-22; for the norm sums of d terms and a root (2^-20 of the row's size) and the
gate's exponential and reciprocal (2^-20)."""
import numpy as np
import pytest

import gret_ref

pytestmark = pytest.mark.gpu
EPS = 1e-5


def f64(t, *shape):
    return None if t is None else t.float().cpu().numpy().astype(np.float64).reshape(*shape)


def norm_case(n, H, d, rms, gate, affine, seed, x=None, in_place=False, pad=0, eps=EPS):
    import torch
    from paper_2405_05254_b200 import binding as yx
    g = torch.Generator().manual_seed(seed)
    W = H * d
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
    buf = rnd(max(n, 1), W + pad) * 3 + 0.5 if x is None else x
    buf = buf.cuda()
    xs = buf[:n, :W]
    gt = rnd(max(n, 1), 2 * W).cuda()[:n, W:] if gate else None
    gain, bias = ((rnd(W) * 0.2 + 1).cuda(), (rnd(W) * 0.1).cuda()) if affine else (None, None)
    want = gret_ref.norm_gate(f64(xs, n, H, d), eps, rms, f64(gt, n, H, d), f64(gain, H, d), f64(bias, H, d)) if n else np.zeros((0, H, d))
    out = buf if in_place else torch.full((n + 1, W + pad), 768.0, dtype=torch.bfloat16, device="cuda")
    ng = yx.make_norm_gate(eps, rms=rms, gate=gt, gain=gain, bias=bias, gate_stride=2 * W)
    yx.yoco_head_norm(yx.HeadNormShape(n, H, d, W + pad, W + pad), xs, ng, out[:n, :W])
    got = f64(out[:n, :W], n, H, d)
    tail = f64(out[n:], -1) if not in_place else np.array([768.0])
    assert (tail == 768.0).all() and (in_place or pad == 0 or bool((out[:n, W:] == 768.0).all()))
    return got, want


@pytest.mark.parametrize("d", [8, 16, 24, 32, 64, 80, 96, 128, 200, 256, 512, 520, 1024])
@pytest.mark.parametrize("rms", [0, 1])
def test_head_norm_sizes(d, rms):
    for n, H, gate, affine in ((1, 1, 1, 0), (37, 3, 1, 1), (5, 16, 0, 0), (130, 2, 0, 1)):
        got, want = norm_case(n, H, d, rms, gate, affine, seed=d + n, pad=8 * (n % 2))
        size = np.abs(want) + 2.0 ** -10               # a value near zero comes from terms of the row's size 1
        assert (np.abs(got - want) <= 2.0 ** -8 * size).all(), (n, H, float((np.abs(got - want) / size).max()))


@pytest.mark.parametrize("d", [40, 48, 56, 72, 104, 136, 160, 168, 248, 320, 328, 640, 648, 768, 776, 1016])
def test_head_norm_lanes_of_a_group(d):
    """Sizes around the borders between the numbers of lanes that share a group, and of pieces that a lane has."""
    for n, H in ((3, 1), (67, 5)):
        got, want = norm_case(n, H, d, 0, 1, 1, seed=d + n)
        assert (np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -10)).all(), (n, H)


def test_head_norm_in_place_empty_and_extreme_rows():
    import torch
    got, want = norm_case(33, 4, 128, 0, 1, 0, seed=1, in_place=True)
    assert (np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -10)).all()
    norm_case(0, 4, 128, 0, 0, 0, seed=1)
    # constant rows: nothing is left of them; a mean far from zero beside a small deviation; tiny and huge rows
    x = torch.zeros(4, 2 * 64)
    x[0] = 3.0
    r = torch.Generator().manual_seed(5)
    x[1] = 1000.0 + torch.randn(128, generator=r) * 16.0
    x[2] = torch.randn(128, generator=r) * 1e-3
    x[3] = torch.randn(128, generator=r) * 1e15
    got, want = norm_case(4, 2, 64, 0, 0, 0, seed=2, x=x.to(torch.bfloat16))
    assert (np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -9)).all() and (got[0] == 0).all()
    got, want = norm_case(4, 2, 64, 1, 0, 0, seed=2, x=x.to(torch.bfloat16))
    assert (np.abs(got - want) <= 2.0 ** -8 * (np.abs(want) + 2.0 ** -10)).all()


def test_gate_far_from_zero():
    """swish far on either side: u itself, and 0 (never NaN)."""
    import torch
    from paper_2405_05254_b200 import binding as yx
    u = torch.tensor([-3e38, -1e4, -200.0, -90.0, -30.0, -5.0, -0.0, 0.0, 1e-30, 5.0, 30.0, 100.0, 1e4, 3e38, 1.0, -1.0] * 4, dtype=torch.bfloat16)
    x = torch.ones(1, 64, dtype=torch.bfloat16)
    y = torch.empty(1, 64, dtype=torch.bfloat16, device="cuda")
    yx.yoco_head_norm(yx.HeadNormShape(1, 1, 64, 0, 0), x.cuda(), yx.make_norm_gate(0.0, rms=True, gate=u.view(1, 64).cuda()), y)
    uf = u.double().numpy()
    with np.errstate(over="ignore"):
        want = uf / (1 + np.exp(-uf))
    got = y.double().cpu().numpy()[0]
    assert np.isfinite(got).all() and (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-24).all()


def rope_case(lens, Hq, Hk, d, rot, pairs, pos, seed, base=640000.0, in_place=False, pad=0):
    import torch
    from paper_2405_05254_b200 import binding as yx
    g = torch.Generator().manual_seed(seed)
    n = int(sum(lens))
    wq, wk = Hq * d, Hk * d
    buf = torch.randn(max(n, 1), wq + wk + pad, generator=g).to(torch.bfloat16).cuda()
    q, k = buf[:n, :wq], buf[:n, wq:wq + wk] if Hk else None
    freq = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    stride = wq + wk + pad
    at = np.concatenate([p + np.arange(m) for p, m in zip(pos, lens)]) if n else np.zeros(0)
    want = [gret_ref.rope(f64(x, n, h, d), at, freq.numpy(), rot, pairs) if x is not None else None for x, h in ((q, Hq), (k, Hk))]
    src = [f64(x, n, h, d) if x is not None else None for x, h in ((q, Hq), (k, Hk))]
    if in_place:
        qr, kr, qs, ks = q, k, stride, stride
    else:
        qo = torch.full((n + 1, wq + 8), 768.0, dtype=torch.bfloat16, device="cuda")
        ko = torch.full((n + 1, wk + 8), 768.0, dtype=torch.bfloat16, device="cuda") if Hk else None
        qr, kr, qs, ks = qo[:n, :wq], ko[:n, :wk] if Hk else None, wq + 8, wk + 8
    shape = yx.make_rope_shape(len(lens), Hq, Hk, d, rot=rot, pairs=pairs, q_stride=stride, k_stride=stride if Hk else 0, q_out_stride=qs,
                               k_out_stride=ks if Hk else 0)
    yx.yoco_rope(shape, q, k, freq.cuda(), np.asarray(pos, np.int32), lens, qr, kr)
    if not in_place:
        for o, w in ((qo, wq), (ko, wk)):
            assert o is None or (bool((o[:, w:] == 768.0).all()) and bool((o[n:] == 768.0).all()))
    for x, y, s, h in ((qr, want[0], src[0], Hq), (kr, want[1], src[1], Hk)):
        if x is None or n == 0:
            continue
        got = f64(x, n, h, d)
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
        size = np.zeros_like(y)
        size[..., a] = size[..., b] = np.abs(s[..., a]) + np.abs(s[..., b])
        # angles: a product and a reduction in 64 bits (2^-51 of the angle), the fraction of a turn rounded to fp32 (2^-25 of a turn)
        tol = 2.0 ** -8 * np.abs(y) + (2.0 ** -20 + 2.0 ** -49 * (at.max() if n else 0)) * size
        assert (np.abs(got - y) <= tol).all(), float((np.abs(got - y) / (tol + 1e-300)).max())
        assert np.array_equal(got[..., rot:], s[..., rot:])


@pytest.mark.parametrize("way", ["norm", "chunk", "step"])
def test_gate_that_closes_against_large_values(way):
    """swish(u) is 0 for u far below zero, and 0 times any finite value is 0, also where u times that value would overflow."""
    import torch
    from paper_2405_05254_b200 import binding as yx
    d, n = 128, 1 if way == "step" else 40
    x = torch.zeros(n, d, dtype=torch.bfloat16, device="cuda")
    x[:, ::8] = 4.0                                          # rms 2^0.5: normalised values 2^1.5; with the gain up to 2^11.5
    gain = torch.full((d,), 1024.0, dtype=torch.bfloat16, device="cuda")
    gate = torch.full((n, d), -3e38, dtype=torch.bfloat16, device="cuda")
    gate[:, 64:] = 1.0
    ng = yx.make_norm_gate(0.0, rms=True, gate=gate, gain=gain)
    y = torch.full((n, d), 768.0, dtype=torch.bfloat16, device="cuda")
    if way == "norm":
        yx.yoco_head_norm(yx.HeadNormShape(n, 1, d, 0, 0), x, ng, y)
    else:
        # k = (1, 0, ..), q = k, no decay before the first token: the first output is v = x, the others multiples of it
        k = torch.zeros_like(x)
        k[:, 0] = 1.0
        state = torch.zeros(1, 1, d, d, device="cuda")
        shape = yx.make_gret_shape(1, 1, d, T=n, scale=1.0)
        slot, begin = np.array([0], np.int32), np.array([-1], np.int32)
        args = (shape, k, k, x, torch.full((n, 1), -0.5, device="cuda"), ng, state, begin, slot)
        if way == "chunk":
            yx.yoco_gret_chunk(*args, None, y, torch.empty(yx.yoco_gret_workspace_size(shape), dtype=torch.uint8, device="cuda"))
        else:
            yx.yoco_gret_step(*args, y)
    got = y.double().cpu().numpy()
    want = np.zeros((n, d))
    want[:, 64::8] = 2 ** 1.5 * 1024 / (1 + np.exp(-1.0))
    # step's and norm's roundings: the output's half step 2^-8; chunk: P and its sum as well, but they leave the norm with the row's size
    assert np.isfinite(got).all() and (np.abs(got - want) <= 2.0 ** -7 * np.abs(want)).all()


@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (128, 32), (80, 16), (80, 80), (112, 96), (512, 512), (16, 16)])
def test_rotation_sizes(d, rot, pairs):
    rope_case([5, 1, 37], 3, 2, d, rot, pairs, [0, 999, 123456], seed=d + rot, pad=8)
    rope_case([70], 1, 0, d, rot, pairs, [17], seed=d + rot + 1)
    rope_case([3, 4], 40, 8, d, rot, pairs, [0, 5], seed=d + rot + 2, in_place=True)


def test_rotation_at_far_positions_and_odd_batches():
    rope_case([40, 3], 2, 1, 128, 128, 0, [1048576, 2 ** 31 - 3], seed=1, base=8e7)
    rope_case([0, 3, 0, 2], 2, 1, 64, 64, 1, [0, 7, 9, 1], seed=2)
    rope_case([0, 0], 2, 1, 64, 64, 1, [0, 7], seed=3)
    rope_case([1] * 512, 2, 2, 64, 64, 0, list(range(0, 512 * 1000, 1000)), seed=4)
    rope_case([2001, 700], 5, 3, 128, 64, 1, [100, 0], seed=5)
    rope_case([3000], 8, 8, 128, 128, 0, [0], seed=6)


def test_a_self_decoders_module_prompt_then_tokens():
    """What a layer runs between its projections: rotation of queries and keys (neighbours, in place), retention with norm and gate over a ragged
    batch of prompts, then single tokens with positions and states advanced in place."""
    import torch
    from paper_2405_05254_b200 import binding as yx
    H, d, lens, extra = 4, 128, [300, 45], 3
    B, W = len(lens), 4 * 128
    g = torch.Generator().manual_seed(9)
    freq = 640000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)
    x = [torch.randn(n + extra, 4 * W + 8, generator=g).to(torch.bfloat16) for n in lens]       # q k v gate z of every sequence
    state = torch.full((B + 1, H, d, d), float("nan"), device="cuda")            # recycled slots: whatever was there
    slots, begin = np.array([2, 0], np.int32), np.array([-1, -1], np.int32)

    prompt = torch.cat([s[:n] for s, n in zip(x, lens)]).cuda()
    cols = lambda t: (t[:, :W], t[:, W:2 * W], t[:, 2 * W:3 * W], t[:, 3 * W:4 * W], t[:, 4 * W:4 * W + H])  # noqa: E731
    stride = 4 * W + 8                                  # (rows start on 16 bytes)
    rs = yx.make_rope_shape(B, H, H, d, T=1, pairs=1, q_stride=stride, k_stride=stride, q_out_stride=stride, k_out_stride=stride)
    sh = yx.make_gret_shape(B, H, d, num_slots=B + 1, tau=16.0, decay_bf16=True, q_stride=stride, k_stride=stride, v_stride=stride, decay_stride=stride)
    q, k, v, gate, z = cols(prompt)
    yx.yoco_rope(rs, q, k, freq.cuda(), np.zeros(B, np.int32), lens, q, k)
    o = torch.empty(sum(lens), W, dtype=torch.bfloat16, device="cuda")
    plain = torch.empty_like(o)
    ws = torch.empty(yx.yoco_gret_workspace_size(sh, lens), dtype=torch.uint8, device="cuda")
    kept = np.array([-1, -1], np.int32)
    yx.yoco_gret_chunk(sh, q, k, v, z, None, state, begin, kept, lens, plain, ws)         # without norm and gate, nothing kept
    ng = yx.make_norm_gate(EPS, rms=True, gate=gate)
    yx.yoco_gret_chunk(sh, q, k, v, z, ng, state, begin, slots, lens, o, ws)
    assert yx.yoco_kv_append_status() == 0
    yx.yoco_head_norm(yx.HeadNormShape(sum(lens), H, d, 0, 0), plain, ng, plain)          # the same in two calls: one rounding more
    assert float((plain.float() - o.float()).norm() / o.float().norm()) < 6e-3

    tok = torch.empty(B, 4 * W + 8, dtype=torch.bfloat16, device="cuda")
    pos = np.array(lens, np.int32)
    tq, tk, tv, tg, tz = cols(tok)
    to = torch.empty(B, W, dtype=torch.bfloat16, device="cuda")
    turn = yx.prepare_tokens("yoco_rope", rs, tq, tk, freq.cuda(), pos, None, tq, tk)
    step = yx.prepare_tokens("yoco_gret_step", sh, tq, tk, tv, tz, yx.make_norm_gate(EPS, rms=True, gate=tg), state, slots, slots, to)
    steps = []
    for t in range(extra):
        tok.copy_(torch.stack([s[n + t] for s, n in zip(x, lens)]))
        turn.run()
        step.run()
        steps.append(to.float().cpu().numpy().copy())
        pos += 1

    at = 0
    for b, n in enumerate(lens):
        rows = x[b].double().numpy()
        N = n + extra
        qd, kd = (gret_ref.rope(rows[:, i * W:(i + 1) * W].reshape(N, H, d), np.arange(N), freq.numpy(), d, 1) for i in (0, 1))
        # the rotated rows are stored in bf16 before the retention reads them
        qd, kd = (torch.from_numpy(a).to(torch.bfloat16).double().numpy() for a in (qd, kd))
        ref, _, end, _ = gret_ref.retention(qd, kd, rows[:, 2 * W:3 * W].reshape(N, H, d), gret_ref.log_decay(rows[:, 4 * W:4 * W + H], 16.0), [N], [None], d ** -0.5)
        y = gret_ref.norm_gate(ref, EPS, 1, rows[:, 3 * W:4 * W].reshape(N, H, d)).reshape(N, W)
        got = np.concatenate([o[at:at + n].float().cpu().numpy()] + [s[b:b + 1] for s in steps])
        assert np.linalg.norm(got - y) <= 6e-3 * np.linalg.norm(y)
        s = state[int(slots[b])].cpu().numpy()
        assert np.linalg.norm(s - end[0]) <= 2e-3 * np.linalg.norm(end[0])      # (a rotated value beside a rounding border may round the other way)
        at += n
    assert bool(torch.isnan(state[1]).all())                                   # nobody's slot


def test_recorded_calls():
    import torch
    from paper_2405_05254_b200 import binding as yx
    x = torch.randn(50, 8 * 128, device="cuda").to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    freq = 1e4 ** (-torch.arange(0, 128, 2, dtype=torch.float64, device="cuda") / 128)
    norm = yx.prepare_tokens("yoco_head_norm", yx.HeadNormShape(50, 8, 128, 0, 0), x, yx.make_norm_gate(EPS), y)
    rope = yx.prepare_tokens("yoco_rope", yx.make_rope_shape(2, 8, 0, 128), y, None, freq, np.array([3, 900], np.int32), [20, 30], z, None)
    norm.run()
    rope.run()
    want = z.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm.run()
        rope.run()
    z.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(z, want)
    del graph
