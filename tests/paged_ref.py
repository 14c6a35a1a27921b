"""Plain numpy forms of the paged-cache operators: caches, rotation, 4-bit rows, attention in 64 bits."""
import numpy as np

import synth_inputs as si

GROUP = 32


def bf16(x):
    """Round fp32 to bf16; returns (bits, the values as fp32)."""
    bits = si.f32_to_bf16_bits(np.asarray(x, np.float32))
    return bits, si.bf16_bits_to_f32(bits)


def cos_sin(max_pos, d, theta=640000.0):
    ang = np.arange(max_pos)[:, None] * theta ** (-np.arange(0, d, 2) / d)
    return np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)


def rotate(x, cs, pairs):
    """fp32 rows [..., d] by table rows cs [..., d]: every operation rounded to fp32 (numpy fuses nothing)."""
    x = np.asarray(x, np.float32)
    half = x.shape[-1] // 2
    c, s = cs[..., :half], cs[..., half:]
    a, b = (x[..., 0::2], x[..., 1::2]) if pairs else (x[..., :half], x[..., half:])
    y = np.empty_like(x)
    y1, y2 = a * c - b * s, b * c + a * s
    if pairs:
        y[..., 0::2], y[..., 1::2] = y1, y2
    else:
        y[..., :half], y[..., half:] = y1, y2
    return y


def quantise(x):
    """fp32 rows [..., d] -> (codes uint8 [..., d/2], scales fp16 [..., d/32]).  A NaN does not count for the scale and is
    stored as the code 1."""
    g = np.asarray(x, np.float32).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    s = np.minimum(np.fmax.reduce(np.abs(g), -1) * np.float32(1.0 / 7.0), np.float32(448)).astype(np.float16)
    with np.errstate(divide="ignore", invalid="ignore"):
        inv = np.where(s > 0, np.float32(1) / s.astype(np.float32), np.float32(0)).astype(np.float32)
        n = np.clip(np.rint(g * inv[..., None]), -7, 7)
    n = (np.where(np.isnan(n), -7, n) + 8).astype(np.uint8).reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    return n[..., 0] | (n[..., 1] << 4), s


def values(codes, s):
    """fp64 values of 4-bit rows."""
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1] // GROUP, GROUP).astype(np.float64)
    return ((n - 8) * s.astype(np.float64)[..., None]).reshape(*codes.shape[:-1], 2 * codes.shape[-1])


class PagedCache:
    """A pool pair with random rows, its page table (unused entries are nonsense) and, per sequence, the rows as fp64."""

    def __init__(self, seed, lens, P, Hkv, d, q4, spare_pages=2, shared=0, gain=1.0, page_rows=0, slack_nan=True):
        r = np.random.default_rng(seed)
        self.lens, self.P, self.Hkv, self.d, self.q4 = np.asarray(lens, np.int32), P, Hkv, d, q4
        per_seq = -(-self.lens // P)
        self.width = max(1, int(per_seq.max()) if len(per_seq) else 1)
        total = int(per_seq.sum()) + spare_pages
        self.num_pages, self.page_rows = total, page_rows or Hkv * P
        order = r.permutation(total).astype(np.int32)
        self.table = r.choice(np.array([-1, total, 2**31 - 1, -2**31], np.int64), (len(lens), self.width)).astype(np.int32)
        at = 0
        for b, n in enumerate(per_seq):
            self.table[b, :n] = order[at:at + n]
            at += n
        if shared:                               # the first `shared` pages of every long enough sequence are those of sequence 0
            for b in range(1, len(lens)):
                k = min(shared, int(per_seq[b]), int(per_seq[0]))
                self.table[b, :k] = self.table[0, :k]
        rows = (total - 1) * self.page_rows + Hkv * P
        live = np.zeros(rows, bool)
        for b, n in enumerate(self.lens):
            for h in range(Hkv):
                live[self.row_numbers(b, h, n)] = True
        self.pools = []
        for which in range(2):
            x = r.standard_normal((rows, d)).astype(np.float32) * (gain if which == 0 else 1.0)
            if q4:
                codes, s = quantise(x)
                if slack_nan:
                    codes[~live] = 0xFF
                    s[~live] = np.nan
                self.pools.append((codes, s))
            else:
                bits, _ = bf16(x)
                if slack_nan:
                    bits[~live] = 0x7FC0
                self.pools.append(bits)

    def row_numbers(self, b, h, n):
        j = np.arange(n)
        return self.table[b, j // self.P].astype(np.int64) * self.page_rows + h * self.P + j % self.P

    def rows(self, which, b, h):
        at = self.row_numbers(b, h, int(self.lens[b]))
        if self.q4:
            codes, s = self.pools[which]
            return values(codes[at], s[at])
        return si.bf16_bits_to_f32(self.pools[which][at]).astype(np.float64)


def attention(cache, Q, T, scale=0.0, window=0):
    """Q [B, Hq, T, d] fp64 -> (O, LSE) by the definition; rows without a visible key give 0 and -inf."""
    B, Hq = Q.shape[:2]
    G = Hq // cache.Hkv
    scale = scale or cache.d ** -0.5
    O, L = np.zeros(Q.shape), np.full(Q.shape[:3], -np.inf)
    for b in range(B):
        n = int(cache.lens[b])
        if n == 0:
            continue
        for h in range(cache.Hkv):
            k, v = cache.rows(0, b, h), cache.rows(1, b, h)
            for g in range(G):
                s = Q[b, h * G + g] @ k.T * scale
                i, j = np.arange(n - T, n)[:, None], np.arange(n)[None, :]
                seen = (j <= i) & ((j > i - window) if window else True)
                s = np.where(seen, s, -np.inf)
                m = s.max(1, keepdims=True)
                e = np.exp(s - np.where(np.isinf(m), 0, m))
                l = e.sum(1, keepdims=True)
                some = l[:, 0] > 0
                O[b, h * G + g, some] = (e @ v)[some] / l[some]
                L[b, h * G + g, some] = (np.where(np.isinf(m), 0, m)[:, 0] + np.log(np.where(l > 0, l, 1))[:, 0])[some]
    return O, L


# ---- on the GPU ---------------------------------------------------------------------------------

def bits_to_dev(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def dev_bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class DevCache:
    def __init__(self, cache, cos_sin=None, pairs=0):
        import torch
        from paper_2405_05254_b200 import binding as bd
        self.cache, self.bd = cache, bd
        if cache.q4:
            self.pools = [torch.from_numpy(a).cuda() for pool in cache.pools for a in pool]       # K4, Ks, V4, Vs
        else:
            self.pools = [bits_to_dev(b) for b in cache.pools]
        self.table = torch.from_numpy(cache.table).cuda()
        self.cos_sin = None if cos_sin is None else torch.from_numpy(cos_sin).cuda()
        self.layout = bd.make_paged_layout(cache.P, cache.num_pages, cache.width, page_rows=cache.page_rows,
                                           cos_sin=self.cos_sin, rope_pairs=pairs)

    def attend(self, Q_bits, T, mode="decode", scale=0.0, window=0, stream=None, ws=None):
        """Returns (O fp64, LSE, O tensor); output buffers carry guard bands."""
        import torch
        from helpers import GUARD, bf16_dev_to_f64
        bd, c = self.bd, self.cache
        B, Hq = Q_bits.shape[:2]
        shape = bd.make_shape(B, Hq, c.Hkv, c.d, T, scale=scale, window=window, max_kv_len=int(c.lens.max()) if B else 0)
        size = bd.yoco_xattn_workspace_size_paged(shape, self.layout, c.lens, bd.MODE_DECODE if mode == "decode" else bd.MODE_CHUNK, c.q4)
        n = B * Hq * T
        o = torch.full((GUARD + n * c.d + GUARD,), 777.0, dtype=torch.bfloat16, device="cuda")
        l = torch.full((GUARD + n + GUARD,), 777.0, dtype=torch.float32, device="cuda")
        w = torch.full((size + 2 * GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
        O, L, W = o[GUARD:GUARD + n * c.d], l[GUARD:GUARD + n], w[GUARD:GUARD + size]
        fn = getattr(bd, f"yoco_xattn_{mode}_paged" + ("_q4" if c.q4 else ""))
        fn(shape, self.layout, bits_to_dev(Q_bits), *self.pools, self.table, c.lens, O, L, W, stream=stream)
        self.status = bd.yoco_xattn_status_detail(W)
        for buf, val in ((o, 777.0), (l, 777.0), (w, 0x5A)):
            assert (buf[:GUARD] == val).all() and (buf[-GUARD:] == val).all(), "guard band overwritten"
        return (bf16_dev_to_f64(O).reshape(B, Hq, T, c.d), L.cpu().numpy().reshape(B, Hq, T), O)
