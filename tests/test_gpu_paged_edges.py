"""The paged cache on the GPU where its operators can go wrong: NaN among ordinary values of a new 4-bit row, peaked scores and
long tails, windows near the end of an int, waits that run out, batches that grow, steps without a token."""
import numpy as np
import pytest

import paged_ref as pr
import synth_inputs as si

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("neighbour", ["ordinary", "clamped"])
@pytest.mark.parametrize("tokens,H,rotated", [(1, 1, False), (19, 2, True), (40, 3, False)])
def test_a_nan_in_a_4_bit_row_is_the_code_1_and_harms_no_other_channel(tokens, H, rotated, neighbour):
    """Bit for bit, whatever else shares the warp: ordinary rows only (no row needs the clamp), or a row that does."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    P, d, lens = 16, 128, np.array([tokens], np.int32)
    cache = pr.PagedCache(71, lens, P, H, d, True, slack_nan=False)
    cs = pr.cos_sin(tokens, d) if rotated else None
    dev = pr.DevCache(cache, cs)
    r = np.random.default_rng(71)
    src = [pr.bf16(r.standard_normal((tokens, H * d)))[0] for _ in range(2)]
    for w, s in enumerate(src):
        for t in range(0, tokens, 2):                                  # every other token has one, or two, somewhere
            s[t, r.integers(0, H * d)] = 0x7FC0
            s[t, (7 * t + 33 * w) % (H * d)] = [0x7FC0, 0xFFC1][w]
        if neighbour == "clamped":
            s[-1, :32] = 0                                             # scale 0
            s[-1, 32:64] = pr.bf16(np.full(32, 3e38, np.float32))[0]   # scale 448
    bd.yoco_paged_append_q4(bd.PagedAppendShape(1, H, d, tokens, 0), dev.layout, pr.bits_to_dev(src[0]), pr.bits_to_dev(src[1]),
                            *dev.pools, dev.table, None, lens)
    assert bd.yoco_kv_append_status() == 0
    for w in range(2):
        codes, s = dev.pools[2 * w].cpu().numpy(), dev.pools[2 * w + 1].cpu().numpy()
        for h in range(H):
            x = si.bf16_bits_to_f32(src[w][:, h * d:(h + 1) * d])
            with np.errstate(invalid="ignore", over="ignore"):
                x = pr.rotate(x, cs, 0) if rotated and w == 0 else x
                want_codes, want_s = pr.quantise(x)
            at = cache.row_numbers(0, h, tokens)
            assert np.array_equal(s[at].view(np.uint16), want_s.view(np.uint16)), (w, h)
            assert np.array_equal(codes[at], want_codes), (w, h)


def test_a_group_of_nothing_but_nan_gets_a_finite_scale():
    """Codes 1 and the largest scale (0 * NaN must not reach the results of rows that do not see this one)."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    cache = pr.PagedCache(72, [5], 16, 1, 128, True, slack_nan=False)
    dev = pr.DevCache(cache)
    x = pr.bf16(np.random.default_rng(72).standard_normal((5, 128)))[0]
    x[2, 64:96] = 0x7FC0
    bd.yoco_paged_append_q4(bd.PagedAppendShape(1, 1, 128, 5, 0), dev.layout, pr.bits_to_dev(x), pr.bits_to_dev(x), *dev.pools, dev.table,
                            None, cache.lens)
    want_codes, want_s = pr.quantise(np.where(np.isnan(si.bf16_bits_to_f32(x)), 0, si.bf16_bits_to_f32(x)))
    want_codes[2, 32:48], want_s[2, 2] = 0x11, np.float16(448)
    at = cache.row_numbers(0, 0, 5)
    for w in range(2):
        assert np.array_equal(dev.pools[2 * w].cpu().numpy()[at], want_codes)
        assert np.array_equal(dev.pools[2 * w + 1].cpu().numpy()[at], want_s)


def q_bits(seed, B, Hq, T, d, gain=1.0):
    return pr.bf16(np.random.default_rng(seed).standard_normal((B, Hq, T, d)) * gain)[0]


def f64(bits):
    return si.bf16_bits_to_f32(bits).astype(np.float64)


@pytest.mark.parametrize("lens,T,P,k_gain,q_gain,window", [
    ([6000], 2, 64, 12.0, 3.0, 0),
    ([2200, 2049], 5, 16, 12.0, 3.0, 0),
    ([6000], 64, 128, 12.0, 3.0, 0),              # two row tiles
    ([6000, 1500, 0, 2047], 40, 32, 4.0, 1.0, 0),
    ([9000], 33, 256, 12.0, 3.0, 4000),
    ([130], 70, 16, 12.0, 3.0, 0),
])
def test_4_bit_chunk_of_peaked_scores(lens, T, P, k_gain, q_gain, window):
    """Scores of some hundreds, a few keys lead every row: there a rounding of K does not average out, however many keys there
    are.  No operand of the scores is rounded: what is left of a score is the fp32 summing of 256 exact products (2^-23 a step of 16, of
    sums up to 2 * 8 s |q| a group, below 3e-4 here), so the log-sum-exp holds the tolerance of the packed cache.  O: its own
    rounding to bf16, half a step 2^-8 of the value (0.0156 where |O| is 4 and more, as the leading keys' values are here: the
    packed cache's tolerance 1e-2 is for outputs below 2.56); V and P rounded to fp16, 2^-11 each, of at most the largest value;
    weights off by twice the scores' 3e-4; the exponentials 2.7e-6."""
    from helpers import assert_lse_close, errors
    cache = pr.PagedCache(17, lens, P, 2, 128, True, gain=k_gain)
    dev = pr.DevCache(cache)
    Q = q_bits(1017, len(lens), 8, T, 128, gain=q_gain)
    o, lse, _ = dev.attend(Q, T, mode="chunk", window=window)
    assert dev.status[0] == 0
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    v = max((np.abs(cache.rows(1, b, h)).max() for b in range(len(lens)) if lens[b] for h in range(2)), default=0.0)
    assert np.isfinite(o).all()
    assert (np.abs(o - ref) <= 2.0 ** -8 * np.abs(ref) + v * (2 * 2.0 ** -11 + 2 * 3e-4 + 2 * 2.7e-6)).all()
    assert errors(o, ref)[1] <= 5e-3
    assert_lse_close(lse, lref, "LSE")


def test_4_bit_decode_and_chunk_agree_on_the_same_cache():
    """Both take the codes and scales as they are: log-sum-exps of up to some hundreds agree to what fp32 sums leave."""
    cache = pr.PagedCache(73, [5000, 700], 64, 2, 128, True, gain=12.0)
    dev = pr.DevCache(cache)
    Q = q_bits(73, 2, 8, 3, 128, gain=3.0)
    lse = [dev.attend(Q, 3, mode=m)[1] for m in ("decode", "chunk")]
    assert np.abs(lse[0].astype(np.float64) - lse[1]).max() <= 2 * 3e-4


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 4, 2**30 + 1, 3])
@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,T,mode", [([2], 8, "decode"), ([2], 8, "chunk"), ([2, 40, 0, 9], 16, "decode"), ([2, 40, 0, 9], 16, "chunk"),
                                         ([1, 300], 200, "chunk")])
def test_windows_as_long_as_an_int_and_more_rows_than_keys(q4, mode, window, lens, T):
    """A window that takes nothing away leaves the plain causal rule, also where the first rows stand before the first key."""
    from helpers import assert_close, assert_lse_close
    cache = pr.PagedCache(74, lens, 16, 2, 128, q4)
    dev = pr.DevCache(cache)
    Q = q_bits(74, len(lens), 2, T, 128)
    o, lse, _ = dev.attend(Q, T, mode=mode, window=window)
    assert dev.status[0] == 0
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,T,P", [([9000, 2500], 16, 1, 64), ([70000], 16, 1, 16), ([30, 0, 7], 8, 2, 32), ([12000] * 3, 32, 2, 256)])
def test_an_expired_wait_of_a_paged_decode_is_reported_and_the_next_call_is_correct(q4, lens, Hq, T, P):
    """Nothing is loaded and the first wait for a tile runs out (limit 20 ms): every CTA leaves, the status names the wait, and the
    same workspace serves the next call."""
    import time
    import torch
    from helpers import assert_close, assert_lse_close, bf16_dev_to_f64
    from paper_2405_05254_b200 import binding as bd
    H = 4
    cache = pr.PagedCache(75, lens, P, H, 128, q4)
    dev = pr.DevCache(cache)
    B = len(lens)
    Qb = q_bits(75, B, Hq, T, 128)
    Q = pr.bits_to_dev(Qb)
    shape = bd.make_shape(B, Hq, H, 128, T)
    ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, dev.layout, cache.lens, bd.MODE_DECODE, q4), dtype=torch.uint8, device="cuda")
    O, L = torch.zeros(B, Hq, T, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hq, T, device="cuda")
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    bd.yoco_xattn_selftest_wait_expiry_paged(shape, dev.layout, Q, dev.pools, dev.table, cache.lens, O, ws, limit_ms=20)
    rc, wait_class, cta = bd.yoco_xattn_status_detail(ws)
    dt = time.perf_counter() - t0
    assert (rc, wait_class) == (bd.ERR_TIMEOUT, bd.WAIT_RING_FULL)
    assert 0 <= cta < 2 * torch.cuda.get_device_properties(0).multi_processor_count
    assert 0.015 < dt < 2.0, dt
    name = "yoco_xattn_decode_paged" + ("_q4" if q4 else "")
    bd.prepare_paged(name, shape, dev.layout, Q, *dev.pools, dev.table, cache.lens, O, L, ws).run()
    assert bd.yoco_xattn_status_detail(ws) == (bd.OK, 0, -1)
    ref, lref = pr.attention(cache, f64(Qb), T)
    assert_close(bf16_dev_to_f64(O).reshape(ref.shape), ref)
    assert_lse_close(L.cpu().numpy(), lref)


@pytest.mark.parametrize("q4", [False, True])
def test_one_workspace_serves_a_batch_while_it_grows(q4):
    """Lengths advanced in place through several ways of cutting the work; the workspace is that of the bound."""
    import torch
    from helpers import assert_close, assert_lse_close, bf16_dev_to_f64
    from paper_2405_05254_b200 import binding as bd
    B, H, steps = 16, 8, [1, 64, 700, 1536, 1537, 2560, 2688]
    cache = pr.PagedCache(76, [steps[-1]] * B, 64, H, 128, q4, slack_nan=False)
    dev = pr.DevCache(cache)
    Qb = q_bits(76, B, H, 1, 128)
    Q = pr.bits_to_dev(Qb)
    shape = bd.make_shape(B, H, H, 128, 1)
    lens = np.full(B, steps[-1], np.int32)
    size = bd.yoco_xattn_workspace_bound_paged(shape, dev.layout, lens, bd.MODE_DECODE, q4)
    buf = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    O, L = torch.empty_like(Q), torch.empty(B, H, 1, device="cuda")
    call = bd.prepare_paged("yoco_xattn_decode_paged" + ("_q4" if q4 else ""), shape, dev.layout, Q, *dev.pools, dev.table, lens, O, L, buf[:size])
    for n in steps:
        lens[:] = n
        lens[3] = n // 2
        call.run()
        assert bd.yoco_xattn_status(buf) == 0
        cache.lens = lens.copy()
        ref, lref = pr.attention(cache, f64(Qb), 1)
        assert_close(bf16_dev_to_f64(O).reshape(ref.shape), ref)
        assert_lse_close(L.cpu().numpy(), lref)
    assert (buf[size:] == 0x5A).all()


@pytest.mark.parametrize("q4", [False, True])
def test_a_step_without_a_token_changes_nothing(q4):
    import torch
    from paper_2405_05254_b200 import binding as bd
    cache = pr.PagedCache(77, [20, 0], 16, 2, 128, q4, slack_nan=False)
    dev = pr.DevCache(cache)
    before = [t.clone() for t in dev.pools]
    none = torch.empty(0, 2 * 128, dtype=torch.bfloat16, device="cuda")
    tail = "_q4" if q4 else ""
    bd.prepare_paged("yoco_paged_append" + tail, bd.PagedAppendShape(2, 2, 128, 0, 0), dev.layout, none, none, *dev.pools, dev.table,
                     np.zeros(2, np.int32), cache.lens).run()
    bd.prepare_paged("yoco_paged_gather" + tail, bd.PagedAppendShape(2, 2, 128, 0, 0), dev.layout, *dev.pools, dev.table, cache.lens, cache.lens,
                     none, none).run()
    assert bd.yoco_kv_append_status() == 0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(before, dev.pools))


@pytest.mark.parametrize("mode", ["chunk", "decode"])
@pytest.mark.parametrize("n,octaves", [(40000, 17.0), (200000, 19.5), (200000, 20.6), (1000000, 21.6)])
def test_4_bit_weights_of_many_keys_behind_one_that_leads_keep_their_bits(mode, n, octaves):
    """All keys are zero but one, which leads by so many octaves and whose value is zero: O is the others' value times their
    share.  Enough streams that most are one CTA's alone, so that the leader sets the maximum of all its keys.  Bound: the
    output's half step 2^-8; P's 2^-11 (it is a normal fp16 number, 2^7 times the weight: 2^-14.6 would be the limit of 21.6
    octaves behind, half a step 2^-25 absolute, 2^-10.4 relative); the row's fp32 sum, 64 keys an addition, each off by half a step 2^-24 of the sum (equal terms do not average
    out): n / 64 * 2^-24, which is the log-sum-exp's error too, beside 2e-5 for the exponentials and fp32 scores; and the chunk
    kernel's sums of n equal products on the tensor core, 16 a step, each step cut at 2^-23 of the sum so far, which is half the
    last one on average: n / 16 * 2^-24."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    B, H, P = 20, 8, 64
    pages = -(-n // P)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].expand(B, pages).contiguous()      # one set of pages for all
    layout = bd.make_paged_layout(P, pages, pages)
    kc = torch.full((pages, H, P, 64), 0x88, dtype=torch.uint8, device="cuda")
    ks = torch.ones(pages, H, P, 4, dtype=torch.float16, device="cuda")
    vc, vs = torch.full_like(kc, 0xCC), torch.full_like(ks, 0.02)
    kc[1, :, 5, 0], vc[1, :, 5] = 0x8F, 0x88                                                               # 7 in channel 0; zeros
    q = pr.bf16(np.array([octaves * np.log(2) / 7 * 128 ** 0.5], np.float32))[1][0]
    Q = torch.zeros(B, H, 1, 128, dtype=torch.bfloat16, device="cuda")
    Q[..., 0] = float(q)
    O, L = torch.empty_like(Q), torch.empty(B, H, 1, device="cuda")
    lens = np.full(B, n, np.int32)
    shape = bd.make_shape(B, H, H, 128, 1)
    ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, layout, lens, bd.MODE_DECODE if mode == "decode" else bd.MODE_CHUNK, True),
                     dtype=torch.uint8, device="cuda")
    bd.prepare_paged(f"yoco_xattn_{mode}_paged_q4", shape, layout, Q, kc, ks, vc, vs, table, lens, O, L, ws).run()
    assert bd.yoco_xattn_status(ws) == 0
    lead = np.exp(float(q) * 7 * 128 ** -0.5)
    want = 4 * float(np.float16(0.02)) * (n - 1) / (n - 1 + lead)
    assert np.abs(O.double().cpu().numpy() / want - 1).max() <= 2.0 ** -8 + 2.0 ** -10.4 + (n / 16 + n / 64) * 2.0 ** -24
    assert np.abs(L.double().cpu().numpy() - np.log(n - 1 + lead)).max() <= n / 64 * 2.0 ** -24 + 2e-5
