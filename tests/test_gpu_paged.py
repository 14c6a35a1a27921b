"""The paged cache on the GPU: append with rotation (bf16 and 4-bit rows), read-back, rotation of the queries, and
decode and chunk attention, against plain numpy (bit for bit where every rounding is fixed by the definition, in 64 bits otherwise).

Tolerances of the attention tests are those of the packed paths (helpers.py).  What the 4-bit path adds: P * s is rounded to
fp16, half a step 2^-11 relative per term, below the bf16 half step 2^-8 that the bf16 path has there; the codes are exact,
the decode scores are fp32 sums of exact products, the chunk path's V values (and K values, with many keys) are rounded to fp16
once (2^-11).  The output's bf16 half step (2^-8) stays the largest single term."""
import numpy as np
import pytest

import paged_ref as pr
import synth_inputs as si
from helpers import assert_close, assert_lse_close

pytestmark = pytest.mark.gpu


def q_bits(seed, B, Hq, T, d, gain=1.0):
    return pr.bf16(np.random.default_rng(seed + 1000).standard_normal((B, Hq, T, d)) * gain)[0]


def f64(bits):
    return si.bf16_bits_to_f32(bits).astype(np.float64)


# ---- append, gather, rope ---------------------------------------------------------------------------

APPEND = [
    # lens (with the new tokens), new tokens, P, Hkv, d, pairs, src_extra, wide pages
    ([1], [1], 16, 1, 128, 0, 0, False),
    ([64, 65, 130], [1, 1, 1], 64, 8, 128, 0, 2048, False),
    ([40, 7, 300], [40, 0, 33], 32, 2, 64, 1, 64, True),
    ([257, 256, 16, 1], [257, 100, 16, 1], 16, 3, 128, 1, 0, False),
    ([512], [301], 256, 4, 128, None, 8, True),
    ([90, 0, 55], [90, 0, 55], 128, 5, 64, 0, 0, False),
    ([3 + i % 37 for i in range(64)], [i % 4 for i in range(64)], 16, 2, 128, 0, 0, False),     # as many as the small table holds
    ([3 + i % 37 for i in range(65)], [i % 4 for i in range(65)], 16, 2, 128, 1, 0, False),     # ... and one more
    ([20] * 512, [1] * 512, 16, 1, 64, 0, 0, False),                                            # as many as a call may have
]


def append_case(case, q4, seed=3):
    import torch
    from paper_2405_05254_b200 import binding as bd
    lens, new, P, H, d, pairs, extra, wide = case
    d = 128 if q4 else d
    lens, new = np.asarray(lens, np.int32), np.asarray(new, np.int32)
    cache = pr.PagedCache(seed, lens, P, H, d, q4, page_rows=2 * H * P if wide else 0, slack_nan=False)
    cs = None if pairs is None else pr.cos_sin(int(lens.max()), d)
    dev = pr.DevCache(cache, cs, pairs or 0)
    tokens, stride = int(new.sum()), H * d + extra
    r = np.random.default_rng(seed)
    src = [pr.bf16(r.standard_normal((tokens, stride)) * np.exp(r.standard_normal((1, stride))))[0] for _ in range(2)]
    if q4:        # rows that reach the corners of the format: zeros, one huge value, tiny values
        for s in src:
            s[0, :32] = 0
            s[0, 32:64] = pr.bf16(np.full(32, 1e-9, np.float32))[0]
            s[-1, 0] = pr.bf16(np.full(1, 3e38, np.float32))[0][0]
            s[-1, 40] = 0x7F80                                             # +inf
    kd, vd = pr.bits_to_dev(src[0]), pr.bits_to_dev(src[1])
    shape = bd.PagedAppendShape(len(lens), H, d, 0, stride)
    fn = bd.yoco_paged_append_q4 if q4 else bd.yoco_paged_append
    fn(shape, dev.layout, kd, vd, *dev.pools, dev.table, new, lens)
    assert bd.yoco_kv_append_status() == 0
    # the same in numpy, in place
    want = [tuple(a.copy() for a in p) if q4 else p.copy() for p in cache.pools]
    at = 0
    for b in range(len(lens)):
        pos = np.arange(lens[b] - new[b], lens[b])
        for h in range(H):
            rows = cache.row_numbers(b, h, int(lens[b]))[pos]
            for which in range(2):
                x = si.bf16_bits_to_f32(src[which][at:at + new[b], h * d:(h + 1) * d])
                if which == 0 and cs is not None:
                    with np.errstate(invalid="ignore", over="ignore"):
                        x = pr.rotate(x, cs[pos], pairs)
                if q4:
                    with np.errstate(invalid="ignore"):
                        want[which][0][rows], want[which][1][rows] = pr.quantise(x)
                else:
                    want[which][rows] = pr.bf16(x)[0]
        at += new[b]
    return cache, dev, want, lens, new, src


@pytest.mark.parametrize("case", APPEND)
def test_append_bf16_bit_for_bit_and_nothing_else_touched(case):
    cache, dev, want, *_ = append_case(case, False)
    for t, w in zip(dev.pools, want):
        assert np.array_equal(pr.dev_bits(t).reshape(w.shape), w)


@pytest.mark.parametrize("case", APPEND)
def test_append_q4_bit_for_bit_and_nothing_else_touched(case):
    cache, dev, want, lens, new, src = append_case(case, True)
    for which in range(2):
        codes, s = dev.pools[2 * which].cpu().numpy(), dev.pools[2 * which + 1].cpu().numpy()
        assert np.array_equal(s.view(np.uint16), want[which][1].view(np.uint16)), "scales"
        assert np.array_equal(codes, want[which][0]), "codes"


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,lo,P,H,d", [([5], [0], 16, 1, 128), ([200, 33, 64], [50, 33, 0], 32, 4, 64), ([300, 1], [299, 0], 256, 3, 128),
                                           ([2 + i % 19 for i in range(70)], [i % 2 for i in range(70)], 16, 2, 128)])
def test_gather_reads_the_rows_back(q4, lens, lo, P, H, d):
    import torch
    from paper_2405_05254_b200 import binding as bd
    d = 128 if q4 else d
    cache = pr.PagedCache(5, lens, P, H, d, q4)
    dev = pr.DevCache(cache)
    lo, hi = np.asarray(lo, np.int32), np.asarray(lens, np.int32)
    n = int((hi - lo).sum()) * H * d
    out = [torch.full((n + 64,), 777.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    fn = bd.yoco_paged_gather_q4 if q4 else bd.yoco_paged_gather
    fn(bd.PagedAppendShape(len(lens), H, d, 0, 0), dev.layout, *dev.pools, dev.table, lo, hi, out[0][:n], out[1][:n])
    assert bd.yoco_kv_append_status() == 0
    for which in range(2):
        want = np.concatenate([np.stack([cache.rows(which, b, h)[lo[b]:] for h in range(H)]).reshape(-1) for b in range(len(lens))])
        assert np.array_equal(pr.dev_bits(out[which][:n]), pr.bf16(want)[0])
        assert (out[which][n:] == 777.0).all()


@pytest.mark.parametrize("pairs", [0, 1])
@pytest.mark.parametrize("B,Hq,T,d,lens", [(1, 1, 1, 64, [1]), (3, 6, 5, 128, [100, 5, 3]), (70, 3, 2, 128, [2 + i for i in range(70)])])
def test_rope_q_bit_for_bit_also_in_place(pairs, B, Hq, T, d, lens):
    import torch
    from paper_2405_05254_b200 import binding as bd
    bits = q_bits(9, B, Hq, T, d)
    cs = pr.cos_sin(120, d)
    table = torch.from_numpy(cs).cuda()
    layout = bd.make_paged_layout(16, 1, 1, cos_sin=table, rope_pairs=pairs)
    Q = pr.bits_to_dev(bits)
    R = torch.empty_like(Q)
    shape = bd.make_shape(B, Hq, 1, d, T)
    bd.yoco_rope_q(shape, layout, Q, np.asarray(lens, np.int32), R)
    want = bits.copy()
    for b in range(B):
        for t in range(T):
            pos = lens[b] - T + t
            if pos >= 0:
                want[b, :, t] = pr.bf16(pr.rotate(si.bf16_bits_to_f32(bits[b, :, t]), cs[pos], pairs))[0]
    assert np.array_equal(pr.dev_bits(R), want)
    bd.yoco_rope_q(shape, layout, Q, np.asarray(lens, np.int32), Q)
    assert np.array_equal(pr.dev_bits(Q), want)


# ---- decode -----------------------------------------------------------------------------------------

DECODE = [
    # lens, Hq, Hkv, T, P, window, d
    ([1], 1, 1, 1, 16, 0, 128),
    ([63, 64, 65], 8, 2, 1, 16, 0, 64),
    ([0, 17, 128], 12, 4, 2, 32, 0, 128),              # an empty sequence; G * T = 6
    ([2, 700], 4, 1, 4, 64, 0, 128),                   # T > N: rows without a key; 16 rows
    ([1000, 31, 513], 32, 8, 1, 128, 100, 128),        # sliding window
    ([5000], 16, 2, 2, 256, 0, 128),                   # 16 rows per KV head
    ([20000, 3000], 32, 8, 1, 64, 0, 128),             # split and merged
    ([4097, 90], 24, 8, 3, 16, 1, 64),                 # window 1: every row sees itself only
    ([9000], 3, 3, 1, 32, 777, 128),
]


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,T,P,window,d", DECODE)
def test_decode_matches_the_definition(q4, lens, Hq, Hkv, T, P, window, d):
    d = 128 if q4 else d
    cache = pr.PagedCache(11, lens, P, Hkv, d, q4)
    dev = pr.DevCache(cache)
    Q = q_bits(11, len(lens), Hq, T, d)
    o, lse, _ = dev.attend(Q, T, window=window)
    assert dev.status[0] == 0
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")


def attention_on_gpu(cache, dev, Q_bits, T):
    """The definition in 64 bits with torch on the GPU, for caches that numpy would take minutes over."""
    import torch
    c = cache
    B, Hq = Q_bits.shape[:2]
    G = Hq // c.Hkv
    Q = pr.bits_to_dev(Q_bits).double()
    O, L = torch.zeros(Q.shape, dtype=torch.float64, device="cuda"), torch.full(Q.shape[:3], -torch.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(c.lens[b])
        seen = torch.arange(n, device="cuda")[None] <= torch.arange(n - T, n, device="cuda")[:, None]
        for h in range(c.Hkv):
            at = torch.from_numpy(c.row_numbers(b, h, n)).cuda()
            rows = []
            for w in range(2):
                if c.q4:
                    codes, s = dev.pools[2 * w][at].int(), dev.pools[2 * w + 1][at].double()
                    x = torch.stack([codes & 15, codes >> 4], -1).reshape(n, c.d).double() - 8
                    rows.append(x * s.repeat_interleave(32, 1))
                else:
                    rows.append(dev.pools[w][at].double())
            for g in range(G):
                s = (Q[b, h * G + g] @ rows[0].T) * c.d ** -0.5
                s = s.masked_fill(~seen, -torch.inf)
                L[b, h * G + g] = torch.logsumexp(s, 1)
                O[b, h * G + g] = torch.softmax(s, 1) @ rows[1]
    return O.cpu().numpy(), L.cpu().numpy()


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,T,P", [
    ([150000, 70001], 8, 8, 1, 16),          # small pages: many batches of page numbers per warp
    ([600000], 16, 8, 2, 64),                # more than 32 tiles per warp of the 4-bit kernel
    ([260000], 32, 4, 2, 32),                # 16 query rows per KV head
    ([700, 1500, 0, 1100, 64], 16, 8, 1, 64),  # whole streams of up to two turns of a CTA's warps
    ([2200, 2300, 1, 900] * 3, 32, 8, 1, 16),  # ... of three turns
    ([1000, 1500], 8, 1, 2, 32),               # ... of two and three turns, 16 query rows
    ([40000, 17, 30000, 0, 5000, 1], 16, 8, 1, 64),     # CTAs that go from stream to stream, some of them empty
    ([9000, 2, 130, 7000, 64, 65, 2500, 12000, 300, 5000, 1111, 640], 12, 4, 2, 16),
])
def test_decode_of_long_caches(q4, lens, Hq, Hkv, T, P):
    cache = pr.PagedCache(47, lens, P, Hkv, 128, q4)
    dev = pr.DevCache(cache)
    Q = q_bits(47, len(lens), Hq, T, 128)
    o, lse, _ = dev.attend(Q, T)
    ref, lref = attention_on_gpu(cache, dev, Q, T)
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")


CHUNK = [
    # lens, Hq, Hkv, T, P, window, d
    ([1], 1, 1, 1, 16, 0, 128),
    ([5, 0, 127], 4, 2, 3, 16, 0, 64),                 # an empty sequence, T > N in none
    ([100, 128, 129], 8, 2, 30, 32, 0, 128),           # 120 rows: the one-tile kernel
    ([300], 12, 4, 50, 64, 0, 128),                    # 150 rows: two tiles
    ([700, 90], 8, 2, 100, 128, 33, 128),              # 400 rows, window; more rows than keys
    ([5000, 1300], 16, 4, 65, 256, 0, 128),            # split and merged
    ([2600], 8, 8, 300, 16, 0, 64),
    ([3001, 40], 32, 8, 40, 16, 0, 128),               # 160 rows per KV head, small pages
    ([4000, 0, 900], 16, 2, 60, 32, 0, 128),           # 2,880 rows in up to 16 pieces: a warp merges a row
    ([2500], 16, 1, 150, 64, 0, 128),                  # 2,400 rows in more pieces than a warp takes
    ([9000, 2000], 4, 1, 9, 64, 500, 128),             # few rows, window, split
]


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,Hkv,T,P,window,d", CHUNK)
def test_chunk_matches_the_definition(q4, lens, Hq, Hkv, T, P, window, d):
    d = 128 if q4 else d
    cache = pr.PagedCache(12, lens, P, Hkv, d, q4)
    dev = pr.DevCache(cache)
    Q = q_bits(12, len(lens), Hq, T, d)
    o, lse, _ = dev.attend(Q, T, mode="chunk", window=window)
    assert dev.status[0] == 0
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")


# lens, Hq, Hkv, T, P, window, mode: rows of few keys (the chunk kernel takes K in two parts there), and both kinds in one call
EXACT_LSE = [
    ([7, 24], 2, 1, 6, 16, 0, "chunk"),
    ([24, 40, 0], 8, 2, 22, 64, 0, "chunk"),
    ([200, 6000], 4, 2, 150, 32, 0, "chunk"),          # one sequence on either side of the rule; a row tile over two heads
    ([700], 4, 4, 600, 256, 0, "chunk"),               # three row tiles of a head, the first with the shortest rows
    ([3000], 4, 1, 40, 128, 70, "chunk"),
    ([3, 40], 6, 2, 3, 16, 0, "decode"),
    ([64, 900], 8, 1, 2, 32, 100, "decode"),
]


@pytest.mark.parametrize("lens,Hq,Hkv,T,P,window,mode", EXACT_LSE)
def test_q4_log_sum_exp_of_few_keys_is_that_of_32_bits(lens, Hq, Hkv, T, P, window, mode):
    """No operand of the scores is rounded, so what is left is: an exponential's relative error (2.7e-6 at most); 16 partial
    products of the tensor core a score (256 channels in two parts), each cut at 2^-23 of the largest sum met, which
    is at most scale * |codes * scale part| . |q| <= 2 scale * 8 s . |q| over a group (the offset of the codes counts: the decode
    kernel adds it as a term of its own); fp32 sums of n weights (n 2^-24); and the fp32 log-sum-exp itself (2^-23).  The sequence of
    6,000 keys takes K rounded to fp16: 2^-11 of a value, at most 2^-11 scale |k| . |q| of its score."""
    cache = pr.PagedCache(15, lens, P, Hkv, 128, True)
    dev = pr.DevCache(cache)
    Q = q_bits(15, len(lens), Hq, T, 128)
    o, lse, _ = dev.attend(Q, T, mode=mode, window=window)
    assert dev.status[0] == 0
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")
    for b, n in enumerate(lens):
        if not n:
            continue
        for h in range(Hkv):
            s = cache.pools[0][1][cache.row_numbers(b, h, n)].astype(np.float64).max(0)          # largest scale per group
            k = np.abs(cache.rows(0, b, h)).max(0)
            for g in range(Hq // Hkv):
                q = np.abs(f64(Q)[b, h * (Hq // Hkv) + g])                                        # [T, 128]
                bound = 2 * 8 * (q.reshape(T, 4, 32).sum(2) @ s) * 128 ** -0.5 * 16 * 2.0 ** -23
                if mode == "chunk" and n >= 2048 and not window:
                    bound += 2.0 ** -11 * (q @ k) * 128 ** -0.5
                bound += 2.7e-6 + n * 2.0 ** -24 + 2.0 ** -23 * np.maximum(1, np.abs(lref[b, h * (Hq // Hkv) + g]))
                got, want = lse[b, h * (Hq // Hkv) + g].astype(np.float64), lref[b, h * (Hq // Hkv) + g]
                seen = ~np.isneginf(want)
                assert (np.abs(got[seen] - want[seen]) <= bound[seen]).all(), (b, h, g, np.abs(got[seen] - want[seen]).max(), bound.min())


@pytest.mark.parametrize("T,d", [(5, 64), (60, 128), (90, 64), (110, 128)])
def test_chunk_bf16_gives_the_bits_of_the_packed_cache(T, d):
    """(Of fewer than 2,048 rows: with more, a paged call's merge may group its sums differently.)"""
    from helpers import GpuRunner
    lens, H, Hq = [1500, 177], 2, 8
    cache = pr.PagedCache(14, lens, 32, H, d, False)
    packed = [np.concatenate([np.concatenate([pr.bf16(cache.rows(w, b, h))[0].reshape(-1) for h in range(H)]) for b in range(len(lens))])
              for w in range(2)]
    Q = q_bits(14, len(lens), Hq, T, d)
    o, lse, O = pr.DevCache(cache).attend(Q, T, mode="chunk")
    po, plse, PO = GpuRunner(len(lens), Hq, H, d, T, lens, packed[0], packed[1]).run(Q, mode="chunk")
    assert np.array_equal(pr.dev_bits(O), pr.dev_bits(PO)) and np.array_equal(lse, plse)


def test_decode_bf16_gives_the_bits_of_the_packed_cache():
    """Same tiles, same plan: a paged cache with the same rows gives the same output bits as the packed one."""
    from helpers import GpuRunner
    lens, H, Hq, d, T = [3000, 77, 1200], 4, 16, 128, 1
    cache = pr.PagedCache(13, lens, 32, H, d, False)
    dev = pr.DevCache(cache)
    packed = [np.concatenate([np.concatenate([pr.bf16(cache.rows(w, b, h))[0].reshape(-1) for h in range(H)]) for b in range(len(lens))])
              for w in range(2)]
    Q = q_bits(13, len(lens), Hq, T, d)
    o, lse, O = dev.attend(Q, T)
    po, plse, PO = GpuRunner(len(lens), Hq, H, d, T, lens, packed[0], packed[1]).run(Q)
    assert np.array_equal(pr.dev_bits(O), pr.dev_bits(PO)) and np.array_equal(lse, plse)


@pytest.mark.parametrize("q4", [False, True])
def test_peaked_scores_and_a_late_maximum(q4):
    """Scores over hundreds: the running maximum moves late, most weights vanish."""
    cache = pr.PagedCache(17, [6000], 64, 2, 128, q4, gain=12.0)
    dev = pr.DevCache(cache)
    Q = q_bits(17, 1, 8, 2, 128, gain=3.0)
    o, lse, _ = dev.attend(Q, 2)
    ref, lref = pr.attention(cache, f64(Q), 2)
    assert_close(o, ref, "O")
    # fp32 scores of some hundreds: their rounding 2^-24 times the sum of |products| (about 128 * 36) is below 3e-4
    assert_lse_close(lse, lref, "LSE")


def test_q4_many_keys_with_small_weights_are_not_lost():
    """One key leads by 12 nats, tens of thousands share the rest: their weights times a small scale are far below the normal
    range of fp16 unless P carries spare bits."""
    n = 40000
    cache = pr.PagedCache(19, [n], 64, 1, 128, True)
    kc, ks = cache.pools[0]
    rows = cache.row_numbers(0, 0, n)
    kc[rows], ks[rows] = 0x88, np.float16(1)                       # every key is zero ...
    x = np.zeros(128, np.float32)
    x[0] = 7
    kc[rows[123]], ks[rows[123]] = pr.quantise(x[None])
    vc, vs = cache.pools[1]
    vc[rows], vs[rows] = 0xCC, np.float16(0.02)                    # ... and every value 4 * 0.02
    vc[rows[123]] = 0x88
    q = np.zeros((1, 1, 1, 128), np.float32)
    q[..., 0] = 12.0 / 7.0 * 128 ** 0.5
    Q = pr.bf16(q)[0]
    o, lse, _ = pr.DevCache(cache).attend(Q, 1)
    ref, lref = pr.attention(cache, f64(Q), 1)
    assert_close(o, ref)
    assert_lse_close(lse, lref)


@pytest.mark.parametrize("q4", [False, True])
def test_pages_shared_by_sequences_and_pools_side_by_side(q4):
    cache = pr.PagedCache(23, [400, 700, 333], 32, 2, 128, q4, shared=5, page_rows=4 * 32 + 32)
    dev = pr.DevCache(cache)
    Q = q_bits(23, 3, 8, 1, 128)
    o, lse, _ = dev.attend(Q, 1)
    ref, lref = pr.attention(cache, f64(Q), 1)
    assert_close(o, ref)
    assert_lse_close(lse, lref)


@pytest.mark.parametrize("q4", [False, True])
def test_pools_of_more_than_2_to_the_32_elements(q4):
    """The pages of a small cache at the far end of a pool pair of 34 million rows: the bits of the small pools' calls."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    H, P, d, T, lens, far = 8, 256, 128, 3, np.array([700, 90], np.int32), 16500
    cache = pr.PagedCache(67, lens, P, H, d, q4, slack_nan=False)
    small = pr.DevCache(cache, pr.cos_sin(1000, d))
    near = bd.make_paged_layout(P, cache.num_pages, cache.width, cos_sin=small.cos_sin)
    big = bd.make_paged_layout(P, far + cache.num_pages, cache.width, cos_sin=small.cos_sin)
    pools = [torch.empty((far + cache.num_pages) * H * P, t.shape[1] if t.dim() > 1 else t.numel() // (cache.num_pages * H * P), dtype=t.dtype,
                         device="cuda") for t in small.pools]
    for t, s in zip(pools, small.pools):
        t[far * H * P:] = s.view(cache.num_pages * H * P, -1)
    table = small.table.clone()
    used = torch.arange(cache.width, device="cuda")[None] < torch.from_numpy(-(-lens // P)).cuda()[:, None]
    table[used] += far
    tail = "_q4" if q4 else ""
    k, v = (torch.randn(4, H * d, device="cuda").to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(2, 16, T, d, device="cuda").to(torch.bfloat16)
    out = []
    for layout, p, t in ((near, small.pools, small.table), (big, pools, table)):
        bd.prepare_paged("yoco_paged_append" + tail, bd.PagedAppendShape(2, H, d, 2, 0), layout, k, v, *p, t, None, lens).run()
        G = [torch.empty(int(lens.sum()) * H * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        bd.prepare_paged("yoco_paged_gather" + tail, bd.PagedAppendShape(2, H, d, 0, 0), layout, *p, t, np.zeros(2, np.int32), lens, *G).run()
        got = G
        for mode in ("decode", "chunk"):
            shape = bd.make_shape(2, 16, H, d, T)
            ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, layout, lens, bd.MODE_DECODE if mode == "decode" else bd.MODE_CHUNK, q4),
                             dtype=torch.uint8, device="cuda")
            O = torch.empty_like(Q)
            bd.prepare_paged(f"yoco_xattn_{mode}_paged{tail}", shape, layout, Q, *p, t, lens, O, None, ws).run()
            assert bd.yoco_xattn_status(ws) == 0
            got.append(O)
        assert bd.yoco_kv_append_status() == 0
        out.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert all(torch.equal(t[far * H * P:].view(torch.uint8), s.view(cache.num_pages * H * P, -1).view(torch.uint8)) for t, s in zip(pools, small.pools))


@pytest.mark.parametrize("mode", ["decode", "chunk"])
@pytest.mark.parametrize("q4", [False, True])
def test_a_bad_page_is_reported_and_harms_nobody_else(q4, mode):
    """Entries outside the pool are read as zeros: the call returns, says BAD_PAGE, the other sequence is right."""
    for bad in (-1, 10**9, -2**31):
        cache = pr.PagedCache(29, [500, 600], 16, 2, 128, q4)
        Q = q_bits(29, 2, 4, 1, 128)
        ref, lref = pr.attention(cache, f64(Q), 1)
        cache.table[0, 7] = bad
        dev = pr.DevCache(cache)
        o, lse, _ = dev.attend(Q, 1, mode=mode)
        assert dev.status[:2] == (dev.bd.ERR_BAD_PAGE, dev.bd.STATUS_BAD_PAGE)
        assert_close(o[1], ref[1])
        assert np.isfinite(o[0]).all()
        cache.table[0, 7] = 0
        dev = pr.DevCache(cache)
        dev.attend(Q, 1, mode=mode)
        assert dev.status[0] == 0                       # the next call starts clean


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("lens,Hq,T,P,window,mode", [
    ([900, 333], 8, 1, 16, 100, "decode"), ([900, 333, 20], 8, 2, 32, 70, "decode"), ([5000], 4, 3, 128, 1, "decode"),
    ([900, 333], 8, 20, 16, 100, "chunk"),                     # 80 rows: the one-tile kernel of the bf16 cache
    ([900, 5000], 8, 90, 32, 130, "chunk"), ([700], 4, 300, 64, 257, "chunk"), ([5000], 4, 9, 256, 1, "chunk"),
])
def test_pages_below_every_window_may_be_gone(q4, lens, Hq, T, P, window, mode):
    """Entries of pages that no row sees any more are nonsense, and unseen rows of the first seen page are NaN."""
    cache = pr.PagedCache(43, lens, P, 2, 128, q4)
    Q = q_bits(43, len(lens), Hq, T, 128)
    ref, lref = pr.attention(cache, f64(Q), T, window=window)
    for b, n in enumerate(lens):
        lo = max(0, n - T + 1 - window)
        for h in range(2):
            at = cache.row_numbers(b, h, lo)
            for pool in cache.pools:
                if q4:
                    pool[0][at], pool[1][at] = 0, np.nan
                else:
                    pool[at] = 0x7FC0 if h else 0x7F80               # NaN, +inf
        cache.table[b, :lo // P] = [-1, 10**9, cache.num_pages][b % 3]
    dev = pr.DevCache(cache)
    o, lse, _ = dev.attend(Q, T, mode=mode, window=window)
    assert dev.status[0] == 0
    assert_close(o, ref, "O")
    assert_lse_close(lse, lref, "LSE")


@pytest.mark.parametrize("q4", [False, True])
def test_append_skips_a_bad_page_and_says_so(q4):
    import torch
    from paper_2405_05254_b200 import binding as bd
    cache = pr.PagedCache(31, [40, 40], 16, 2, 128, q4, slack_nan=False)
    cache.table[1, 2] = cache.num_pages
    dev = pr.DevCache(cache)
    before = [t.clone() for t in dev.pools]
    x = pr.bits_to_dev(q_bits(31, 1, 1, 2, 256).reshape(2, 256))
    fn = bd.yoco_paged_append_q4 if q4 else bd.yoco_paged_append
    fn(bd.PagedAppendShape(2, 2, 128, 1, 0), dev.layout, x, x, *dev.pools, dev.table, None, cache.lens)
    assert bd.yoco_kv_append_status_detail()[:2] == (bd.ERR_BAD_PAGE, bd.STATUS_BAD_PAGE)
    assert bd.yoco_kv_append_status() == 0
    changed = [(a.view(cache.num_pages * 2 * 16, -1) != b.view(cache.num_pages * 2 * 16, -1)).any(1).sum().item()
               for a, b in zip(before, dev.pools)]
    assert all(c == 2 for c in changed), changed         # the two heads of the one good row


@pytest.mark.parametrize("q4", [False, True])
def test_a_recorded_step_follows_the_page_table_and_two_streams_do_not_meet(q4):
    import torch
    from paper_2405_05254_b200 import binding as bd
    caches = [pr.PagedCache(37 + i, [900, 150], 64, 2, 128, q4) for i in range(2)]
    devs = [pr.DevCache(c) for c in caches]
    Qb = [q_bits(37 + i, 2, 8, 1, 128) for i in range(2)]
    calls, outs, streams, graphs = [], [], [torch.cuda.Stream() for _ in range(2)], []
    for i in range(2):
        c, dev = caches[i], devs[i]
        shape = bd.make_shape(2, 8, 2, 128, 1)
        ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, dev.layout, c.lens, bd.MODE_DECODE, q4), dtype=torch.uint8, device="cuda")
        O = torch.empty(2 * 8 * 128, dtype=torch.bfloat16, device="cuda")
        name = "yoco_xattn_decode_paged" + ("_q4" if q4 else "")
        call = bd.prepare_paged(name, shape, dev.layout, pr.bits_to_dev(Qb[i]), *dev.pools, dev.table, c.lens, O, None, ws, stream=streams[i])
        torch.cuda.synchronize()
        call.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[i]):
            call.run()
        calls.append(call), outs.append(O), graphs.append(g)
    # the second sequence moves to other pages: same rows, other places
    refs = [pr.attention(caches[i], f64(Qb[i]), 1)[0] for i in range(2)]
    dev, c = devs[0], caches[0]
    old, new = int(c.table[1, 0]), int(np.setdiff1d(np.arange(c.num_pages), np.concatenate([c.table[0, :15], c.table[1, :3]]))[0])
    R = 2 * 64
    for t in dev.pools:
        v = t.view(c.num_pages, R, -1)
        v[new] = v[old]
        v[old] = 255 if t.dtype == torch.uint8 else float("nan")
    dev.table[1, 0] = new
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    from helpers import bf16_dev_to_f64
    for i in range(2):
        assert_close(bf16_dev_to_f64(outs[i]).reshape(refs[i].shape), refs[i])


@pytest.mark.parametrize("q4", [False, True])
def test_a_prepared_call_follows_its_lengths_and_the_current_stream(q4):
    """kv_len is read at every run(), numbers of new tokens are those of the preparation, and run() goes to the stream that
    is current then (a call given a stream stays on it)."""
    import torch
    from helpers import bf16_dev_to_f64
    from paper_2405_05254_b200 import binding as bd
    H, Hq, P, steps = 2, 8, 16, 5
    tail = "_q4" if q4 else ""
    lens = np.array([30, 63], np.int32)
    cache = pr.PagedCache(53, lens + steps, P, H, 128, q4, slack_nan=False)
    dev = pr.DevCache(cache)
    dev.layout.page_rows = cache.page_rows
    new, B = np.array([1, 1], np.int32), 2
    shape = bd.make_shape(B, Hq, H, 128, 1)
    r = np.random.default_rng(53)
    x = torch.empty(B, 2 * H * 128, dtype=torch.bfloat16, device="cuda")
    Q, O = torch.empty(B, Hq, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(B, Hq, 1, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, dev.layout, lens + steps, bd.MODE_DECODE, q4) + 4096, dtype=torch.uint8, device="cuda")
    store = bd.prepare_paged("yoco_paged_append" + tail, bd.PagedAppendShape(B, H, 128, 0, 2 * H * 128), dev.layout, x[:, :H * 128],
                             x[:, H * 128:], *dev.pools, dev.table, new, lens)
    attend = bd.prepare_paged("yoco_xattn_decode_paged" + tail, shape, dev.layout, Q, *dev.pools, dev.table, lens, O, None, ws)
    new[:] = 10**6                                        # not read again
    shape.T, dev.layout.num_pages = 50, 1                 # neither are these
    side = torch.cuda.Stream()
    for step in range(steps):
        lens += 1
        src = pr.bf16(r.standard_normal((B, 2 * H * 128)))[0]
        Qb = q_bits(60 + step, B, Hq, 1, 128)
        for b in range(B):
            for h in range(H):
                at = cache.row_numbers(b, h, int(lens[b]))[-1]
                for w in range(2):
                    y = si.bf16_bits_to_f32(src[b, (w * H + h) * 128:(w * H + h + 1) * 128])[None]
                    if q4:
                        cache.pools[w][0][at], cache.pools[w][1][at] = (a[0] for a in pr.quantise(y))
                    else:
                        cache.pools[w][at] = pr.bf16(y)[0][0]
        xd, qd = pr.bits_to_dev(src), pr.bits_to_dev(Qb)
        torch.cuda.synchronize()
        with torch.cuda.stream(side if step % 2 else torch.cuda.current_stream()):
            torch.cuda._sleep(2_000_000)                  # about a millisecond: a call on another stream would be too early
            x.copy_(xd.view_as(x))
            Q.copy_(qd.view_as(Q))
            store.run()
            attend.run()
        torch.cuda.synchronize()
        cache.lens = lens.copy()
        assert_close(bf16_dev_to_f64(O), pr.attention(cache, f64(Qb), 1)[0])


@pytest.mark.parametrize("q4", [False, True])
def test_a_recorded_prompt_step_and_the_same_bits_every_time(q4):
    """Append, rotation and chunk attention in one graph, replayed with other rows, other queries and other pages, give the
    bits of the calls made one by one; repeated calls give the same bits."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    H, Hq, P, T, B = 2, 8, 32, 70, 2
    tail = "_q4" if q4 else ""
    lens = np.array([1900, 70], np.int32)
    cache = pr.PagedCache(59, lens, P, H, 128, q4, spare_pages=70, slack_nan=False)
    dev = pr.DevCache(cache, pr.cos_sin(2000, 128), 1)
    shape, rows = bd.make_shape(B, Hq, H, 128, T), bd.PagedAppendShape(B, H, 128, T, 0)
    k, v = (torch.randn(B * T, H * 128, device="cuda").to(torch.bfloat16) for _ in range(2))
    Q = torch.randn(B, Hq, T, 128, device="cuda").to(torch.bfloat16)
    R, O, L = torch.empty_like(Q), torch.empty_like(Q), torch.empty(B, Hq, T, device="cuda")
    ws = torch.empty(bd.yoco_xattn_workspace_size_paged(shape, dev.layout, lens, bd.MODE_CHUNK, q4), dtype=torch.uint8, device="cuda")
    calls = [bd.prepare_paged("yoco_paged_append" + tail, rows, dev.layout, k, v, *dev.pools, dev.table, None, lens),
             bd.prepare_paged("yoco_rope_q", shape, dev.layout, Q, lens, R),
             bd.prepare_paged("yoco_xattn_chunk_paged" + tail, shape, dev.layout, R, *dev.pools, dev.table, lens, O, L, ws)]

    def step():
        for c in calls:
            c.run()

    def result():
        torch.cuda.synchronize()
        assert bd.yoco_xattn_status(ws) == 0 and bd.yoco_kv_append_status() == 0
        return [t.clone().view(torch.uint8) for t in (O, L, *dev.pools)]

    step()
    first = result()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for t in (O, L):
        t.fill_(7.0)
    for _ in range(3):
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(), first))
    k.normal_(), v.normal_(), Q.normal_()
    spare = np.setdiff1d(np.arange(cache.num_pages), np.concatenate([cache.table[0], cache.table[1, :3]]))
    dev.table[0, :60] = torch.from_numpy(spare[:60].astype(np.int32)).cuda()          # pages with other rows
    g.replay()
    replayed = result()
    assert not torch.equal(replayed[0], first[0])
    O.fill_(7.0)
    step()
    assert all(torch.equal(a, b) for a, b in zip(result(), replayed))


@pytest.mark.parametrize("lens,Hq,T,P,mode", [([70000, 9], 16, 1, 16, "decode"), ([30000] * 3, 32, 2, 64, "decode"), ([9000, 130], 8, 70, 128, "chunk")])
@pytest.mark.parametrize("q4", [False, True])
def test_the_same_call_gives_the_same_bits(q4, lens, Hq, T, P, mode):
    cache = pr.PagedCache(61, lens, P, 4, 128, q4)
    dev = pr.DevCache(cache)
    Q = q_bits(61, len(lens), Hq, T, 128)
    runs = [dev.attend(Q, T, mode=mode) for _ in range(6)]
    for o, lse, _ in runs[1:]:
        assert np.array_equal(o, runs[0][0]) and np.array_equal(lse, runs[0][1])


@pytest.mark.parametrize("q4", [False, True])
def test_a_serving_run_append_rotate_attend_step_by_step(q4):
    """Tokens arrive one by one and in a chunk, keys and queries are rotated by one table, every step is attended over the
    cache so far; the plain form quantises (or rounds) the same rows and evaluates the definition."""
    import torch
    from paper_2405_05254_b200 import binding as bd
    H, Hq, d, P, B = 2, 8, 128, 16, 3
    steps = [([40, 3, 17], 40), ([1, 1, 1], 1), ([2, 2, 2], 2), ([1, 1, 1], 1)]
    final = np.sum([s[0] for s in steps], 0)
    cache = pr.PagedCache(41, final, P, H, d, q4)
    cs = pr.cos_sin(64, d)
    dev = pr.DevCache(cache, cs)
    r = np.random.default_rng(41)
    lens = np.zeros(B, np.int32)
    for new, _ in steps:
        new = np.asarray(new, np.int32)
        lens = (lens + new).astype(np.int32)
        src = [pr.bf16(r.standard_normal((int(new.sum()), H * d)))[0] for _ in range(2)]
        fn = bd.yoco_paged_append_q4 if q4 else bd.yoco_paged_append
        fn(bd.PagedAppendShape(B, H, d, 0, 0), dev.layout, pr.bits_to_dev(src[0]), pr.bits_to_dev(src[1]), *dev.pools, dev.table, new, lens)
        at = 0
        for b in range(B):
            pos = np.arange(lens[b] - new[b], lens[b])
            for h in range(H):
                rows = cache.row_numbers(b, h, int(lens[b]))[pos]
                for w in range(2):
                    x = si.bf16_bits_to_f32(src[w][at:at + new[b], h * d:(h + 1) * d])
                    x = pr.rotate(x, cs[pos], 0) if w == 0 else x
                    if q4:
                        cache.pools[w][0][rows], cache.pools[w][1][rows] = pr.quantise(x)
                    else:
                        cache.pools[w][rows] = pr.bf16(x)[0]
            at += new[b]
        T = int(new.min())
        if T > 2:
            continue                                        # the prompt is only stored
        cache.lens = lens
        Q = q_bits(41, B, Hq, T, d)
        shape = bd.make_shape(B, Hq, H, d, T)
        Qd = pr.bits_to_dev(Q)
        bd.yoco_rope_q(shape, dev.layout, Qd, lens, Qd)
        Qr = pr.dev_bits(Qd)
        o, lse, _ = dev.attend(Qr, T)
        ref, lref = pr.attention(cache, f64(Qr), T)
        assert_close(o, ref)
        assert_lse_close(lse, lref)
    assert bd.yoco_kv_append_status() == 0
