"""The paged-cache operators: what is measured, their plain forms, and their definition in 64 bits.

A paged cache holds rows of ``d`` channels, one per (page, KV head, slot): row = page * page_rows + head * P + slot.
``page_table[b, j]`` names the page that holds positions [j P, (j + 1) P) of sequence ``b``.  Two element formats:

* ``bf16``: pools ``[pages, Hkv, P, d]``;
* ``q4``: codes ``[pages, Hkv, P, d / 2]`` (channel 2 i in the low nibble of byte i, 2 i + 1 in the high one) and fp16
  scales ``[pages, Hkv, P, d / 32]``; a value is (code - 8) * scale, codes 1..15.

Operators: ``append`` (rotate the new keys by their positions and store keys and values; for q4 the rows are then read
back as the values they stand for), ``decode`` (a few query rows per KV head over the whole cache) and ``chunk`` (any
number of new rows, causal).
"""
import numpy as np
import torch

own = False

GROUP = 32          # channels that share a scale of a 4-bit row
SCALE_MAX = 448.0   # largest scale a 4-bit row is given


def _case(name, op, fmt, B, T, lens, P, d=128, Hq=32, Hkv=8, window=0, pairs=0, spread=0):
    return {"name": name, "op": op, "fmt": fmt, "B": B, "T": T, "len": lens, "spread": spread, "P": P, "d": d, "Hq": Hq,
            "Hkv": Hkv, "window": window, "pairs": pairs}


def listed():
    """``len``/``spread``: the sequences' lengths lie spread over [len, len + spread], dealt out by the seed.  For append, ``T``
    is the most new tokens of a sequence; with ``spread`` > 0 they bring different numbers, from 1 to T."""
    return [
        # one decode step of a batch of 64: the new token of every sequence, keys and that layer's queries rotated
        _case("append bf16 one token x 64", "append", "bf16", 64, 1, 900, 64, spread=6000),
        # a ragged prompt chunk into small pages, rotation on neighbouring channels
        _case("append bf16 ragged prompt", "append", "bf16", 5, 2041, 2100, 16, spread=2500, pairs=1),
        # one decode step into a 4-bit cache
        _case("append q4 one token x 37", "append", "q4", 37, 1, 300, 32, spread=4000),
        # prompt chunks of 16K tokens into a 4-bit cache
        _case("append q4 prompt", "append", "q4", 8, 2048, 2048, 64, spread=1000),
        # a short conversation, one user: launch latency
        _case("decode bf16 one short", "decode", "bf16", 1, 1, 513, 16),
        # sixteen ragged sequences, the usual serving batch
        _case("decode bf16 ragged x 16", "decode", "bf16", 16, 1, 1000, 64, spread=31000),
        # one sequence of 1M keys: the long-context step
        _case("decode bf16 1M", "decode", "bf16", 1, 1, 1048576, 256),
        # a few short sequences in 4 bits
        _case("decode q4 short x 8", "decode", "q4", 8, 1, 700, 64, spread=400),
        # sixteen ragged sequences in 4 bits, two query rows each (one drafted token)
        _case("decode q4 ragged x 16", "decode", "q4", 16, 2, 4001, 32, spread=60000),
        # 1M keys in 4 bits
        _case("decode q4 1M", "decode", "q4", 1, 1, 1048576, 64),
        # two prompt chunks of 512 tokens behind a cached prefix
        _case("chunk bf16 512 x 2", "chunk", "bf16", 2, 512, 33280, 64),
        # a prompt chunk behind a long 4-bit prefix, odd sizes
        _case("chunk q4 391", "chunk", "q4", 1, 391, 65927, 128),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "chunk"])
    fmt = rng.choice(["bf16", "q4"])
    d = 128 if fmt == "q4" else rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8])
    G = rng.choice([1, 2, 3, 4, 8])
    P = rng.choice([16, 32, 64, 128, 256])
    c = {"op": op, "fmt": fmt, "d": d, "Hkv": Hkv, "Hq": Hkv * G, "P": P, "window": 0, "pairs": rng.choice([0, 1])}
    if op == "append":
        c["B"] = _log(rng, 1, 96)
        c["T"] = rng.choice([1, 1, 2, _log(rng, 3, max(4, 16000 // c["B"]))])
        c["len"] = c["T"] + _log(rng, 1, 1500)
        c["spread"] = rng.choice([0, _log(rng, 10, 3000)])
    elif op == "decode":
        c["B"] = _log(rng, 1, 48)
        c["T"] = rng.choice([t for t in (1, 1, 2, 3, 4) if G * t <= 16])
        c["len"] = c["T"] + _log(rng, 1, 400000 // c["B"])
        c["spread"] = rng.choice([0, c["len"] // 2])
        c["window"] = rng.choice([0, 0, 0, _log(rng, 64, 2048)])
    else:
        c["B"] = rng.choice([1, 1, 2, 3])
        c["T"] = _log(rng, 5, 400)
        c["len"] = c["T"] + _log(rng, 1, 30000 // c["B"])
        c["spread"] = rng.choice([0, c["len"] // 3])
        c["window"] = rng.choice([0, 0, _log(rng, 64, 2048)])
    return c


# ---- inputs -------------------------------------------------------------------------------------

def _lengths(case, seed):
    """Lengths and numbers of new tokens: the case fixes the set (spread over its range), the seed who has which."""
    B = case["B"]
    r = np.random.RandomState(seed % (1 << 31))
    part = (np.arange(B) * 0.6180339887498949) % 1.0
    n = case["len"] + np.round(case["spread"] * part / max(part.max(), 1e-9)).astype(np.int64)
    new = np.full(B, case["T"])
    if case["op"] == "append" and case["spread"]:
        new = 1 + np.round((case["T"] - 1) * (1.0 - part)).astype(np.int64)
    return n[r.permutation(B)].astype(np.int32), new[r.permutation(B)].astype(np.int32)


def _quantise(x):
    """fp32 [..., d] -> codes uint8 [..., d / 2], scales fp16 [..., d / 32]."""
    g = x.reshape(*x.shape[:-1], -1, GROUP)
    s = (g.abs().amax(-1) * (1.0 / 7.0)).clamp(max=SCALE_MAX).half()
    inv = torch.where(s > 0, s.float().reciprocal(), torch.zeros((), device=x.device))
    n = (torch.round(g * inv[..., None]).clamp(-7, 7) + 8).to(torch.uint8).reshape(*x.shape[:-1], -1, 2)
    return n[..., 0] | (n[..., 1] << 4), s


def _values(codes, s):
    """The fp32 values that 4-bit rows stand for."""
    n = torch.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1, GROUP)
    return ((n.float() - 8.0) * s.float()[..., None]).reshape(*codes.shape[:-1], -1)


def _pool(case, gen, pages, per_channel):
    """One pool of cached rows: normal values, for keys with a few strong channels (as trained models have them)."""
    B, H, P, d = case["B"], case["Hkv"], case["P"], case["d"]
    gain = torch.exp(0.4 * torch.randn(H, 1, d, generator=gen, device="cuda")) if per_channel else torch.ones(H, 1, d, device="cuda")
    step = max(1, (1 << 26) // (H * P * d))
    if case["fmt"] == "bf16":
        pool = torch.empty(pages, H, P, d, dtype=torch.bfloat16, device="cuda")
        for i in range(0, pages, step):
            n = min(step, pages - i)
            pool[i:i + n] = torch.randn(n, H, P, d, generator=gen, device="cuda") * gain
        return pool
    codes = torch.empty(pages, H, P, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(pages, H, P, d // GROUP, dtype=torch.float16, device="cuda")
    for i in range(0, pages, step):
        n = min(step, pages - i)
        codes[i:i + n], scales[i:i + n] = _quantise(torch.randn(n, H, P, d, generator=gen, device="cuda") * gain)
    return codes, scales


def prepare(case, seed):
    B, T, H, Hq, P, d = (case[k] for k in ("B", "T", "Hkv", "Hq", "P", "d"))
    kv_len, new = _lengths(case, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    per_seq = -(-kv_len // P)
    width, used = int(per_seq.max()), int(per_seq.sum())
    pages = used + 3                                        # a few pages belong to nobody
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    slot = torch.full((B, width), -1, dtype=torch.int64)
    first = np.concatenate([[0], np.cumsum(per_seq)])
    for b in range(B):
        slot[b, :per_seq[b]] = torch.arange(int(first[b]), int(first[b + 1]))
    slot = slot.cuda()
    table = torch.where(slot >= 0, order[slot.clamp(min=0)], torch.full((), -1, dtype=torch.int32, device="cuda")).contiguous()
    st = {"case": dict(case), "kv_len": kv_len, "new": new, "table": table, "pages": pages,
          "K": _pool(case, gen, pages, True), "V": _pool(case, gen, pages, False)}
    if case["op"] == "append":
        n_tok, max_pos = int(new.sum()), int(kv_len.max())
        qkv = torch.randn(n_tok, 2 * H * d, generator=gen, device="cuda").to(torch.bfloat16)   # the projection's output
        st["k_new"], st["v_new"] = qkv[:, :H * d], qkv[:, H * d:]
        freq = 640000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        ang = torch.arange(max_pos, device="cuda", dtype=torch.float64)[:, None] * freq
        st["cos_sin"] = torch.cat((ang.cos(), ang.sin()), -1).float().contiguous()
        if T == 1:
            st["Q"] = torch.randn(B, Hq, T, d, generator=gen, device="cuda").to(torch.bfloat16)
            st["Qr"] = torch.empty_like(st["Q"])
        # where every new token goes (what a program with plain operations keeps beside its batch)
        st["seq"] = torch.from_numpy(np.repeat(np.arange(B), new)).cuda()
        st["pos"] = torch.from_numpy(np.concatenate([np.arange(n - m, n) for n, m in zip(kv_len, new)])).cuda()
        if case["fmt"] == "q4":
            st["Kb"] = torch.empty(H * n_tok * d, dtype=torch.bfloat16, device="cuda")
            st["Vb"] = torch.empty_like(st["Kb"])
    else:
        st["Q"] = torch.randn(B, Hq, T, d, generator=gen, device="cuda").to(torch.bfloat16)
        st["len_dev"] = torch.from_numpy(kv_len).cuda()
        st["O"] = torch.empty_like(st["Q"])
        st["lse"] = torch.empty(B, Hq, T, dtype=torch.float32, device="cuda")
    if own:
        _plan(st)
    return st


# ---- the framework's calls ----------------------------------------------------------------------

def _plan(st):
    """The layout, workspace and marshalled calls that a serving loop keeps."""
    from paper_2405_05254_b200 import binding as yx
    c = st["case"]
    B, T, H, Hq, P, d = (c[k] for k in ("B", "T", "Hkv", "Hq", "P", "d"))
    q4 = c["fmt"] == "q4"
    tail = "_q4" if q4 else ""
    pools = (*st["K"], *st["V"]) if q4 else (st["K"], st["V"])
    layout = yx.make_paged_layout(P, st["pages"], st["table"].shape[1], cos_sin=st.get("cos_sin"), rope_pairs=c["pairs"])
    if c["op"] == "append":
        shape = yx.PagedAppendShape(B, H, d, T, st["k_new"].stride(0))
        st["calls"] = [yx.prepare_paged("yoco_paged_append" + tail, shape, layout, st["k_new"], st["v_new"], *pools,
                                        st["table"], st["new"], st["kv_len"])]
        if q4:
            st["calls"].append(yx.prepare_paged("yoco_paged_gather_q4", shape, layout, *pools, st["table"],
                                                st["kv_len"] - st["new"], st["kv_len"], st["Kb"], st["Vb"]))
        if T == 1:
            st["calls"].append(yx.prepare_paged("yoco_rope_q", yx.make_shape(B, Hq, H, d, T), layout, st["Q"], st["kv_len"],
                                                st["Qr"]))
        return
    mode = yx.MODE_DECODE if c["op"] == "decode" else yx.MODE_CHUNK
    shape = yx.make_shape(B, Hq, H, d, T, max_kv_len=int(st["kv_len"].max()), window=c["window"])
    ws = torch.empty(yx.yoco_xattn_workspace_size_paged(shape, layout, st["kv_len"], mode, q4), dtype=torch.uint8, device="cuda")
    st["calls"] = [yx.prepare_paged("yoco_xattn_%s_paged%s" % (c["op"], tail), shape, layout, st["Q"], *pools, st["table"],
                                    st["kv_len"], st["O"], st["lse"], ws)]


# ---- plain forms --------------------------------------------------------------------------------

def _rotate(x, cs, pairs):
    """fp32 rows [..., d] by their angles [..., d] (cosines, then sines)."""
    cos, sin = cs.chunk(2, -1)
    x1, x2 = (x[..., 0::2], x[..., 1::2]) if pairs else x.chunk(2, -1)
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    return torch.stack((y1, y2), -1).flatten(-2) if pairs else torch.cat((y1, y2), -1)


def _append_plain(st):
    c = st["case"]
    H, P, d = c["Hkv"], c["P"], c["d"]
    pos, seq = st["pos"], st["seq"]
    page, slot = st["table"][seq, pos // P].long(), pos % P
    cs = st["cos_sin"][pos]
    k = _rotate(st["k_new"].float().view(-1, H, d), cs[:, None], c["pairs"])
    v = st["v_new"].float().view(-1, H, d)
    out = {}
    if c["fmt"] == "bf16":
        st["K"][page, :, slot] = k.to(torch.bfloat16)
        st["V"][page, :, slot] = v.to(torch.bfloat16)
        out["K"], out["V"] = st["K"], st["V"]
    else:
        for name, x in (("K", k), ("V", v)):
            codes, scales = _quantise(x)
            st[name][0][page, :, slot] = codes
            st[name][1][page, :, slot] = scales
            rows = _values(st[name][0][page, :, slot], st[name][1][page, :, slot]).to(torch.bfloat16)   # [tokens, H, d]
            # packed head-major: [H, new_i, d] per sequence
            new = torch.bincount(seq, minlength=c["B"])
            begin = torch.cumsum(new, 0) - new
            t = torch.arange(len(seq), device="cuda") - begin[seq]
            at = (begin[seq] * H)[:, None] + torch.arange(H, device="cuda") * new[seq][:, None] + t[:, None]
            st[name + "b"].view(-1, d)[at] = rows
            out[name] = st[name + "b"]
    if c["T"] == 1:
        out["Q"] = _rotate(st["Q"].float(), cs[:, None, None], c["pairs"]).to(torch.bfloat16)
    return out


def _attend_plain(st):
    c = st["case"]
    B, T, H, Hq, P, d = (c[k] for k in ("B", "T", "Hkv", "Hq", "P", "d"))
    at = st["table"].long().clamp(min=0)

    def rows(pool):                                               # [B, H, width * P, d] fp32
        x = _values(pool[0][at], pool[1][at]) if c["fmt"] == "q4" else pool[at].float()
        return x.transpose(1, 2).reshape(B, H, -1, d)

    q = st["Q"].float().view(B, H, Hq // H * T, d)
    s = q @ rows(st["K"]).transpose(-1, -2)
    s *= d ** -0.5
    n = st["len_dev"].long()[:, None, None, None]
    j = torch.arange(s.shape[-1], device="cuda")
    i = n - T + torch.arange(T, device="cuda").repeat(Hq // H)[:, None]
    seen = (j <= i) & (j < n)
    if c["window"]:
        seen &= j > i - c["window"]
    v = rows(st["V"])
    v.masked_fill_((j >= n[:, :, 0])[..., None], 0.0)             # slots behind a sequence may hold anything
    s.masked_fill_(~seen, float("-inf"))
    m = s.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    s -= m
    s.exp_()
    l = s.sum(-1, keepdim=True)
    o = (s @ v) / torch.where(l > 0, l, torch.ones_like(l))
    return {"O": o.view(B, Hq, T, d).to(torch.bfloat16), "lse": (m + l.log()).view(B, Hq, T)}


def run(st):
    op = st["case"]["op"]
    if not own:
        return _append_plain(st) if op == "append" else _attend_plain(st)
    for call in st["calls"]:
        call.run()
    if op != "append":
        return {"O": st["O"], "lse": st["lse"]}
    out = {"K": st["Kb"], "V": st["Vb"]} if "Kb" in st else {"K": st["K"], "V": st["V"]}
    if "Qr" in st:
        out["Q"] = st["Qr"]
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------

def _row_bytes(case):
    return case["d"] * 2 if case["fmt"] == "bf16" else case["d"] // 2 + case["d"] // GROUP * 2


def work(case):
    B, T, H, Hq, d = (case[k] for k in ("B", "T", "Hkv", "Hq", "d"))
    row = _row_bytes(case)
    lens, new = _lengths(case, 0)
    n = float(lens.mean())
    if case["op"] == "append":
        tok = int(new.sum())
        moved = tok * (2 * H * d * 2 + d * 4 + 2 * H * row)
        if case["fmt"] == "q4":                                    # read back: rows in, bf16 out
            moved += tok * 2 * H * (row + d * 2)
        if T == 1:
            moved += B * Hq * d * 4
        return {"bytes": moved, "flops": tok * H * d * 3}
    keys = n if not case["window"] else min(n, case["window"] + T - 1)
    seen = min(n, case["window"]) if case["window"] else max(n - (T - 1) / 2, 1)
    return {"bytes": B * (keys * 2 * H * row + Hq * T * (4 * d + 4) + keys / case["P"] * 4),
            "flops": 4.0 * B * Hq * T * d * seen}


# ---- the definition in 64 bits ----------------------------------------------------------------------

def _rows64(case, pool, table_row, head, n):
    """Rows [n, d] of one sequence and KV head, by flat row numbers."""
    P, H = case["P"], case["Hkv"]
    j = torch.arange(n, device="cuda")
    flat = table_row.long()[j // P] * (H * P) + head * P + j % P
    if case["fmt"] == "bf16":
        return pool.view(-1, case["d"])[flat].double()
    byte = pool[0].view(-1, case["d"] // 2)[flat].int()
    scale = pool[1].view(-1, case["d"] // GROUP)[flat].double()
    out = torch.empty(n, case["d"], dtype=torch.float64, device="cuda")
    out[:, 0::2] = (byte % 16 - 8).double()
    out[:, 1::2] = (byte // 16 - 8).double()
    return out * scale.repeat_interleave(GROUP, 1)


def _turn64(x, ang, pairs):
    """x [..., d] in 64 bits as complex numbers times cos + i sin."""
    half = x.shape[-1] // 2
    c = torch.complex(ang[..., :half].double(), ang[..., half:].double())
    z = torch.view_as_complex(x.reshape(*x.shape[:-1], half, 2).contiguous()) if pairs else torch.complex(x[..., :half], x[..., half:])
    z = z * c
    return torch.view_as_real(z).reshape(x.shape) if pairs else torch.cat((z.real, z.imag), -1)


def exact(case, seed):
    st = prepare(case, seed)
    B, T, H, Hq, P, d = (case[k] for k in ("B", "T", "Hkv", "Hq", "P", "d"))
    out = {}
    if case["op"] == "append":
        at = np.concatenate([[0], np.cumsum(st["new"])])
        for name, src in (("K", st["k_new"]), ("V", st["v_new"])):
            pool = st[name].double() if case["fmt"] == "bf16" else None
            packed = []
            for b in range(B):
                lo, hi = int(at[b]), int(at[b + 1])
                x = src[lo:hi].double().reshape(hi - lo, H, d)
                pos = torch.arange(int(st["kv_len"][b]) - (hi - lo), int(st["kv_len"][b]), device="cuda")
                if name == "K":
                    x = _turn64(x, st["cos_sin"][pos][:, None].expand(-1, H, -1), case["pairs"])
                if pool is not None:
                    flat = st["table"][b].long()[pos // P] * (H * P) + pos % P
                    for h in range(H):
                        pool.view(-1, d)[flat + h * P] = x[:, h]
                else:
                    g = x.reshape(hi - lo, H, d // GROUP, GROUP)
                    s = torch.clamp(g.abs().amax(-1) / 7, max=SCALE_MAX).half().double()
                    n = torch.clamp(torch.round(g / torch.where(s > 0, s, torch.ones_like(s))[..., None]), -7, 7)
                    packed.append((n * s[..., None]).reshape(hi - lo, H, d).transpose(0, 1).reshape(-1))
            out[name] = pool if pool is not None else torch.cat(packed)
        if T == 1:
            pos = torch.from_numpy(st["kv_len"].astype(np.int64) - 1).cuda()
            out["Q"] = _turn64(st["Q"].double(), st["cos_sin"][pos][:, None, None].expand(-1, Hq, T, -1), case["pairs"])
        return out
    G = Hq // H
    o = torch.zeros(B, Hq, T, d, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq, T), float("-inf"), dtype=torch.float64, device="cuda")
    for b in range(B):
        n = int(st["kv_len"][b])
        for h in range(H):
            k, v = (_rows64(case, st[x], st["table"][b], h, n) for x in ("K", "V"))
            for t0 in range(0, T, 64):
                t1 = min(T, t0 + 64)
                hi = torch.arange(n - T + t0, n - T + t1, device="cuda")[:, None]
                key = torch.arange(n, device="cuda")
                see = (key <= hi) & (key > hi - case["window"]) if case["window"] else key <= hi
                for g in range(G):
                    q = st["Q"][b, h * G + g, t0:t1].double()
                    x = torch.where(see, q @ k.T / d ** 0.5, torch.full((), -torch.inf, dtype=torch.float64, device="cuda"))
                    z = torch.logsumexp(x, 1)
                    lse[b, h * G + g, t0:t1] = z
                    o[b, h * G + g, t0:t1] = torch.exp(x - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None]) @ v
    return {"O": o, "lse": lse}
