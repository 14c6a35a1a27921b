"""Gated retention on the GPU against its recurrence in 64 bits: prompts (token by token and in chunks on the tensor cores, whole streams and
cut ones), single tokens, states in slots, the output's norm and gate.

Tolerances.  A rounding to bf16 is off by at most 2^-8 of the value (half a step; 2^-9 where the value is not just above a power of
two).  O (no norm): one for the output, relative to the output; in the chunks one for P and one for the copy of the state, relative to the sums of
magnitudes (o_abs), which bound both: |O - o| <= 2^-8 |o| + 2^-8 o_abs, and in the 2-norm over a whole call the independent roundings
give 3 * 1.7e-3 at most (5e-3 is asked).  The state: products and sums in fp32 (2^-24 each, a handful per token), decays to 2^-22
each, over the tokens that still weigh: 1e-5 of the sums of magnitudes for decays whose memory is up to a few hundred tokens."""
import numpy as np
import pytest

import gret_ref

pytestmark = pytest.mark.gpu

GUARD = 64          # elements around outputs that have to stay


class Problem:
    def __init__(self, lens, H, d, tau=16.0, seed=0, norm=None, fused=True, decay_dtype=None, slots=None, fresh=(), logs=None, scale=0.0, states=1.0,
                 gain=False, bias=False, in_place=False):
        import torch
        self.torch, self.lens, self.H, self.d, self.tau, self.norm = torch, list(lens), H, d, tau, norm
        B, n, W = len(lens), int(sum(lens)), H * d
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
        x = rnd(max(n, 1), 4 * W).cuda()
        if fused:
            self.q, self.k, self.v, self.gate = (x[:n, i * W:(i + 1) * W] for i in range(4))
        else:
            self.q, self.k, self.v, self.gate = (x[:n, i * W:(i + 1) * W].contiguous() for i in range(4))
        if logs is not None:
            z = torch.as_tensor(logs, dtype=torch.float32).reshape(n, H)
        elif tau:
            z = torch.randn(n, H, generator=g) * 1.5 + 1.0
        else:
            z = -torch.rand(n, H, generator=g) * 2.0 ** -(torch.arange(H) % 7).float()
        self.decay = z.to(decay_dtype or torch.float32).cuda()
        self.n_slots = 2 * B + 1
        perm = torch.randperm(self.n_slots, generator=g).numpy().astype(np.int32) if slots is None else np.asarray(slots, np.int32)
        self.slot_in = perm[:B].copy()
        self.slot_out = self.slot_in.copy() if in_place else perm[B:2 * B].copy()
        for i in fresh:
            self.slot_in[i] = -1
        self.state = (torch.randn(self.n_slots, H, d, d, generator=g) * states).cuda()
        self.state0 = self.state.cpu().numpy().copy()
        self.gain = (rnd(W) * 0.2 + 1).cuda() if gain else None
        self.bias = (rnd(W) * 0.1).cuda() if bias else None
        self.scale = scale
        self.o_buf = torch.full((n + 2, W + GUARD), 768.0, dtype=torch.bfloat16, device="cuda")
        self.o = self.o_buf[1:n + 1, :W]
        stride = lambda t: t.stride(0) if n > 1 else 0  # noqa: E731
        from paper_2405_05254_b200 import binding as yx
        self.yx = yx
        self.shape = yx.make_gret_shape(B, H, d, T=1, num_slots=self.n_slots, scale=scale, tau=tau, decay_bf16=self.decay.dtype == torch.bfloat16,
                                        q_stride=stride(self.q), k_stride=stride(self.k), v_stride=stride(self.v), o_stride=W + GUARD)
        self.ng = None if norm is None else yx.make_norm_gate(1e-5, rms=norm == "rms", gate=self.gate, gain=self.gain, bias=self.bias,
                                                              gate_stride=stride(self.gate))

    def workspace(self):
        n = self.yx.yoco_gret_workspace_size(self.shape, self.lens)
        return self.torch.full((n + 512,), 0xA5, dtype=self.torch.uint8, device="cuda"), n

    def chunk(self):
        ws, n = self.workspace()
        self.yx.yoco_gret_chunk(self.shape, self.q, self.k, self.v, self.decay, self.ng, self.state, self.slot_in, self.slot_out, self.lens, self.o, ws[:n])
        assert self.yx.yoco_kv_append_status() == 0
        assert bool((ws[n:] == 0xA5).all()), "behind the workspace"
        return self

    def step(self):
        self.yx.yoco_gret_step(self.shape, self.q, self.k, self.v, self.decay, self.ng, self.state, self.slot_in, self.slot_out, self.o)
        return self

    def reference(self):
        H, d = self.H, self.d
        f = lambda t: t.float().cpu().numpy().astype(np.float64).reshape(-1, H, d)  # noqa: E731
        states = [None if s < 0 else self.state0[s] for s in self.slot_in]
        scale = self.scale or d ** -0.5
        logs = gret_ref.log_decay(self.decay.float().cpu().numpy(), self.tau)
        o, o_abs, out, out_abs = gret_ref.retention(f(self.q), f(self.k), f(self.v), logs, self.lens, states, scale)
        return o, o_abs, out, out_abs

    def check(self):
        torch = self.torch
        o, o_abs, out, out_abs = self.reference()
        n, H, d = len(o), self.H, self.d
        got = self.o.float().cpu().numpy().astype(np.float64).reshape(n, H, d)
        buf = self.o_buf.float().cpu().numpy()
        assert (buf[0] == 768.0).all() and (buf[-1] == 768.0).all() and (buf[:, H * d:] == 768.0).all(), "around the output"
        if n:
            assert np.isfinite(got).all()
            if self.norm is None:
                tol = 2.0 ** -8 * np.abs(o) + 2.0 ** -8 * o_abs + 1e-30
                assert (np.abs(got - o) <= tol).all(), float((np.abs(got - o) / tol).max())
                ref = o
            else:
                f = lambda t, *s: None if t is None else t.float().cpu().numpy().astype(np.float64).reshape(*s)  # noqa: E731
                ref = gret_ref.norm_gate(o, 1e-5, self.norm == "rms", f(self.gate, n, H, d), f(self.gain, H, d), f(self.bias, H, d))
            assert np.linalg.norm(got - ref) <= 5e-3 * np.linalg.norm(ref)
        pool = self.state.cpu().numpy().astype(np.float64)
        want = self.state0.astype(np.float64)
        for i, s in enumerate(self.slot_out):
            if s >= 0:
                err = np.abs(pool[s] - out[i])
                assert (err <= 1e-5 * out_abs[i] + 1e-30).all(), (i, float((err / (out_abs[i] + 1e-30)).max()))
                want[s] = pool[s]
        assert np.array_equal(pool, want), "a slot that is nobody's"
        return got


LENS = [[1], [2], [7, 1, 24], [25], [127], [128], [129], [1, 64, 300, 128], [31, 0, 257, 0], [700, 40, 5]]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", LENS, ids=str)
def test_prompts_against_the_recurrence(lens, d):
    Problem(lens, 3, d, tau=16.0, seed=len(lens)).chunk().check()


@pytest.mark.parametrize("d", [64, 128])
def test_streams_are_cut_when_there_are_few(d):
    import torch
    p = Problem([1500], 2, d, tau=16.0, seed=3)
    assert p.workspace()[1] > 0                             # two streams of 12 chunks: cut over 24 CTAs
    p.chunk().check()
    # whole streams (as many as the device has SMs and more): no workspace
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert p.yx.yoco_gret_workspace_size(p.yx.make_gret_shape(sms, 1, d, T=300), None) == 0
    Problem([150] * 40, 4, d, seed=4).chunk().check()
    Problem([300, 26, 140] * 20, 3, d, seed=5, in_place=True).chunk().check()


@pytest.mark.parametrize("d", [64, 128])
def test_ranges_of_chunks_that_hold_several_streams(d):
    """Few streams, more chunks than SMs: a CTA's range begins and ends inside streams and has whole ones, and last chunks, in between."""
    p = Problem([2600, 777, 3, 1900], 6, d, seed=6, norm="group")
    assert p.workspace()[1] > 0
    p.chunk().check()
    Problem([130] * 9 + [9000], 5, d, seed=7, in_place=True).chunk().check()


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_start_on_16_bytes(d):
    """Output and gate may start on any 16 bytes; rows that start on 32 go another way."""
    import torch
    for lens in ([300, 25], [200] * 3):
        p = Problem(lens, 2, d, seed=8, norm="rms")
        n, W = sum(lens), 2 * d
        p.o_buf = torch.full((n + 2, W + 40), 768.0, dtype=torch.bfloat16, device="cuda")
        p.o = p.o_buf[1:n + 1, :W]
        gate = torch.zeros(n, W + 24, dtype=torch.bfloat16, device="cuda")
        gate[:, 8:8 + W] = p.gate
        p.gate = gate[:, 8:8 + W]
        assert p.o.data_ptr() % 32 == 16 and p.gate.data_ptr() % 32 == 16
        p.shape.o_stride = W + 40
        p.ng = p.yx.make_norm_gate(1e-5, rms=True, gate=p.gate, gate_stride=W + 24)
        p.chunk().check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kw", [dict(tau=0.0), dict(tau=0.0, fused=False), dict(tau=1.0), dict(tau=16.0, decay_dtype="bfloat16"), dict(scale=0.7, fresh=(0, 2)),
                                dict(in_place=True), dict(fresh=(0, 1, 2), in_place=True)], ids=str)
def test_forms_of_decays_slots_and_rows(kw, d):
    import torch
    kw = dict(kw)
    if "decay_dtype" in kw:
        kw["decay_dtype"] = getattr(torch, kw["decay_dtype"])
    Problem([40, 300, 17], 2, d, seed=11, **kw).chunk().check()
    Problem([9, 3, 17], 2, d, seed=12, **kw).chunk().check()
    Problem([1, 1, 1], 5, d, seed=13, **kw).step().check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", ["group", "rms"])
@pytest.mark.parametrize("affine", [0, 1])
def test_norm_and_gate_of_the_output(norm, affine, d):
    kw = dict(norm=norm, gain=bool(affine), bias=bool(affine))
    Problem([300, 17], 2, d, seed=21, **kw).chunk().check()
    Problem([5, 24], 2, d, seed=22, **kw).chunk().check()
    Problem([1] * 4, 3, d, seed=23, **kw).step().check()


@pytest.mark.parametrize("d", [64, 128])
def test_strong_decays_beside_weak_ones(d):
    """A token that forgets everything, tokens that forget nearly everything, and weak decays behind them: what is behind must not feel the size of
    the sums before it."""
    n, H = 300, 2
    r = np.random.RandomState(5)
    logs = -0.002 * r.rand(n, H)
    logs[r.randint(0, n, 25), :] = -100.0
    logs[r.randint(0, n, 6), :] = -1e4
    logs[77] = -np.inf
    logs[128:150] = -60.0
    Problem([n], H, d, tau=0.0, logs=logs, seed=31).chunk().check()
    Problem([20], H, d, tau=0.0, logs=logs[70:90], seed=32).chunk().check()
    z = np.where(r.rand(n, H) < 0.1, -3e4, 30.0)            # logits: saturated on both sides
    Problem([n], H, d, tau=16.0, logs=z, seed=33).chunk().check()
    Problem([1, 1], H, d, tau=16.0, logs=np.array([[-np.inf, 1e30], [np.inf, -1e30]]), seed=34).step().check()


@pytest.mark.parametrize("d", [64, 128])
def test_no_decay_at_all_sums_everything(d):
    n, H = 400, 2
    Problem([n], H, d, tau=0.0, logs=np.zeros((n, H)), seed=41, states=0.0).chunk().check()


@pytest.mark.parametrize("d", [64, 128])
def test_rows_behind_a_sequence_do_not_reach_it(d):
    """The last chunk of a sequence brings rows of the next one, which may hold anything."""
    p = Problem([200, 130, 90], 2, d, seed=51)
    lo, hi = 200, 330
    for t in (p.q, p.k, p.v):
        t[lo:hi] = float("nan")
    p.decay[lo:hi] = float("nan")
    p.chunk()
    o, o_abs, out, _ = p.reference()
    got = p.o.float().cpu().numpy().astype(np.float64).reshape(o.shape)
    for a, b in ((0, 200), (330, 420)):
        assert (np.abs(got[a:b] - o[a:b]) <= 2.0 ** -8 * (np.abs(o[a:b]) + o_abs[a:b])).all()
    pool = p.state.cpu().numpy()
    assert np.isfinite(pool[p.slot_out[0]]).all() and np.isfinite(pool[p.slot_out[2]]).all() and np.isnan(pool[p.slot_out[1]]).any()


def test_a_prompt_in_pieces_and_token_by_token_is_the_same_prompt():
    """One call, two calls, one call and single tokens: the state goes from call to call (chunkwise, token by token, step)."""
    H, d = 4, 128
    whole = Problem([330], H, d, seed=61, in_place=True)
    yx, W = whole.yx, H * d
    ref = whole.state.clone()
    whole.chunk()
    o, end = whole.o.float().clone(), whole.state.clone()
    for cuts in ([200, 130], [300, 14, 16], [325, 1, 1, 1, 1, 1]):
        whole.state.copy_(ref)
        whole.o.zero_()
        t = 0
        for n in cuts:
            a = [x[t:t + n] for x in (whole.q, whole.k, whole.v, whole.decay)]
            sh = yx.make_gret_shape(1, H, d, T=n, num_slots=whole.n_slots, tau=16.0, q_stride=4 * W, k_stride=4 * W, v_stride=4 * W, o_stride=W + GUARD)
            if n == 1:
                yx.yoco_gret_step(sh, *a, None, whole.state, whole.slot_in, whole.slot_in, whole.o[t:t + n])
            else:
                ws = whole.torch.empty(yx.yoco_gret_workspace_size(sh), dtype=whole.torch.uint8, device="cuda")
                yx.yoco_gret_chunk(sh, *a, None, whole.state, whole.slot_in, whole.slot_in, None, whole.o[t:t + n], ws)
            t += n
        s = int(whole.slot_in[0])
        assert float((whole.state[s] - end[s]).norm() / end[s].norm()) < 5e-6
        assert float((whole.o.float() - o).norm() / o.norm()) < 6e-3


def test_a_shared_prefix_and_states_that_are_not_kept():
    """Several sequences start from one slot; a state that goes nowhere, zero-length sequences that hand theirs on."""
    for lens in ([150, 40, 200, 0, 0], [3, 2, 9, 0, 0]):
        p = Problem(lens, 2, 128, seed=71)
        p.slot_in[:] = [4, 4, 4, 4, -1]
        p.slot_out[:] = [0, -1, 2, 7, 9]
        p.chunk().check()


def test_recorded_calls_and_calls_on_another_stream():
    import torch
    for lens in ([400, 60], [12, 3], [200] * 30):
        p = Problem(lens, 4, 128, seed=81, norm="rms", in_place=False)
        ws = torch.empty(p.yx.yoco_gret_workspace_size(p.shape, p.lens), dtype=torch.uint8, device="cuda")
        call = p.yx.prepare_tokens("yoco_gret_chunk", p.shape, p.q, p.k, p.v, p.decay, p.ng, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
        call.run()
        torch.cuda.synchronize()
        want, end = p.o.clone(), p.state.clone()
        side = torch.cuda.Stream()
        p.o.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call.run()
        side.synchronize()
        assert torch.equal(p.o, want) and torch.equal(p.state, end)              # the same bits
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call.run()
        for _ in range(3):
            p.o.zero_()
            p.state[torch.as_tensor(p.slot_out.astype(np.int64))] = 5.0
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(p.o, want) and torch.equal(p.state, end)
        del graph


def test_cut_streams_recorded_in_a_row_and_at_once():
    """The three kernels of cut streams start early behind one another, but never ahead of the call before: one workspace serves calls in a row, in a
    recorded graph too, and two streams with a workspace each do not meet."""
    import torch
    ps = [Problem([2100, 900], 3, d, seed=97 + d, norm="group", in_place=True) for d in (64, 128)]
    wss = [torch.empty(p.workspace()[1], dtype=torch.uint8, device="cuda") for p in ps]
    assert all(ws.numel() > 0 for ws in wss)
    calls = [p.yx.prepare_tokens("yoco_gret_chunk", p.shape, p.q, p.k, p.v, p.decay, p.ng, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
             for p, ws in zip(ps, wss)]
    start = [p.state.clone() for p in ps]
    want = []
    for p, call in zip(ps, calls):
        for _ in range(4):                                   # each goes on from the state that the one before left
            call.run()
            torch.cuda.synchronize()
        want.append((p.o.clone(), p.state.clone()))

    def begin():
        for p, s0 in zip(ps, start):
            p.o.zero_()
            p.state.copy_(s0)
        torch.cuda.synchronize()

    def same():
        torch.cuda.synchronize()
        for p, (o, s) in zip(ps, want):
            assert torch.equal(p.o, o) and torch.equal(p.state, s)

    begin()
    for call in calls:
        for _ in range(4):
            call.run()
    same()
    begin()
    sides = [torch.cuda.Stream() for _ in ps]
    for _ in range(4):
        for call, side in zip(calls, sides):
            with torch.cuda.stream(side):
                call.run()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in calls:
            for _ in range(4):
                call.run()
    for _ in range(3):
        begin()
        graph.replay()
        same()
    del graph


def test_two_calls_at_once():
    import torch
    ps = [Problem([700, 260], 6, d, seed=90 + d) for d in (64, 128)]
    wss = [p.workspace()[0] for p in ps]
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for _ in range(5):
        for p, ws, st in zip(ps, wss, streams):
            with torch.cuda.stream(st):
                p.yx.yoco_gret_chunk(p.shape, p.q, p.k, p.v, p.decay, None, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
    torch.cuda.synchronize()
    for p in ps:
        p.check()


def test_many_sequences():
    """More sequences than the small table holds, and the most there may be."""
    for B, hi in ((65, 40), (512, 30), (512, 3)):
        r = np.random.RandomState(B + hi)
        Problem(r.randint(0, hi, B), 1, 64, seed=B, in_place=True).chunk().check()
    Problem([1] * 512, 2, 64, seed=7).step().check()


def test_a_workspace_for_other_lengths_is_refused():
    import torch
    from paper_2405_05254_b200 import binding as yx
    p = Problem([1500], 2, 128, seed=95)
    n = yx.yoco_gret_workspace_size(p.shape, p.lens)
    for ws in (None, torch.empty(n - 16, dtype=torch.uint8, device="cuda")):
        with pytest.raises(yx.YocoError) as e:
            yx.yoco_gret_chunk(p.shape, p.q, p.k, p.v, p.decay, None, p.state, p.slot_in, p.slot_out, p.lens, p.o, ws)
        assert e.value.code == (yx.ERR_INVALID_ARG if ws is None else yx.ERR_WORKSPACE_TOO_SMALL)
