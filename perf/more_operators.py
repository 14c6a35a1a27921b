"""The operators of a self-decoder with gated retention: what is measured, their plain forms, and their definition in 64 bits.

Per head, with queries q_t, keys k_t, values v_t of ``d`` channels and a decay g_t in (0, 1], a state S of ``d`` x ``d`` runs along a sequence:

    S_t = g_t S_(t-1) + k_t^T v_t,   o_t = scale q_t S_t

* ``chunk``: whole prompts or chunks of them, ragged, each from a state of the pool (or from zero) into a state of the pool;
* ``step``: one token of every sequence;
* ``norm``: each head's output normalised over its channels and gated, y = swish(gate) * (o - mean) / sqrt(var + eps) (or by its
  root mean square); chunk and step take it along where a case says so;
* ``rope``: queries and keys turned by the angles of their positions, as they come out of the projection (token after token).

``gate``d decays are logits z of g = sigmoid(z)^(1 / tau); otherwise they are natural logarithms of g.
"""
import numpy as np
import torch

own = False

TAU = 16.0
EPS = 1e-5


def _chunk(name, B, lo, hi, H, d, tau=TAU, fused=1, norm=0, fresh=0):
    return {"name": name, "op": "chunk", "B": B, "lo": lo, "hi": hi, "H": H, "d": d, "tau": tau, "fused": fused, "norm": norm, "fresh": fresh}


def _step(name, B, H, d, tau=TAU, fused=1, norm=0, fresh=0):
    return {"name": name, "op": "step", "B": B, "lo": 1, "hi": 1, "H": H, "d": d, "tau": tau, "fused": fused, "norm": norm, "fresh": fresh}


def _norm(name, tokens, H, d, rms=0, affine=0, gate=1):
    return {"name": name, "op": "norm", "B": 1, "lo": tokens, "hi": tokens, "H": H, "d": d, "rms": rms, "affine": affine, "gate": gate}


def _rope(name, B, lo, hi, Hq, Hk, d, rot, pairs, pos, base=640000.0, stretch=1.0):
    return {"name": name, "op": "rope", "B": B, "lo": lo, "hi": hi, "H": Hq, "Hk": Hk, "d": d, "rot": rot, "pairs": pairs, "pos": pos, "base": base,
            "stretch": stretch}


def listed():
    """``lo``..``hi``: tokens of a sequence, spread over the range and dealt out by the seed.  ``fused``: q, k and v are slices of one
    projection.  ``norm``: 1 group norm and gate, 2 the same by the root mean square.  ``fresh``: every ``fresh``-th sequence begins here."""
    return [
        # a few drafted tokens of every sequence of a small batch, verified at once: latency and states
        _chunk("chunk 5 drafted x 16", 16, 5, 5, 8, 128),
        # a ragged batch of short prompts, small heads, some of them beginning
        _chunk("chunk ragged x 6", 6, 37, 1501, 16, 64, norm=2, fresh=2),
        # one long prompt's next piece
        _chunk("chunk 4096", 1, 4096, 4096, 32, 128, norm=2),
        # a whole prompt of odd length from nothing
        _chunk("chunk 32719", 1, 32719, 32719, 32, 128, tau=0.0, fused=0, fresh=1),
        # one user's next token
        _step("step x 1", 1, 32, 128, norm=2),
        # a serving batch's next tokens
        _step("step x 64", 64, 32, 128, norm=2),
        # the same with small heads and fixed decays, nothing fused
        _step("step d64 x 37", 37, 24, 64, tau=0.0, fused=0, fresh=5),
        # the heads' outputs of one decode step
        _norm("norm 64 tokens", 64, 32, 128, rms=1),
        # the heads' outputs of a prompt, groups of an odd size, gain and bias
        _norm("norm 16001 tokens", 16001, 40, 80, affine=1),
        # one decode step at far positions
        _rope("rope one token x 64", 64, 1, 1, 32, 8, 128, 128, 0, 1000000),
        # a ragged batch of prompt chunks, half of every head turned, neighbouring channels, positions stretched
        _rope("rope ragged x 5", 5, 301, 4099, 16, 16, 128, 64, 1, 30000, stretch=4.0),
        # a whole prompt
        _rope("rope 32768", 1, 32768, 32768, 32, 32, 128, 128, 1, 0, base=8e7),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    case = _draw(rng)
    del case["name"]
    return case


def _draw(rng):
    op = rng.choice(["chunk", "chunk", "step", "norm", "rope"])
    d = rng.choice([64, 128, 128])
    tau, fused, norm, fresh = rng.choice([0.0, TAU]), rng.choice([0, 1]), rng.choice([0, 0, 1, 2]), rng.choice([0, 1, 2, 3])
    if op == "chunk":
        B, H = _log(rng, 1, 24), rng.choice([1, 3, 8, 16, 24, 32])
        hi = _log(rng, 1, max(2, 800000 // (B * H)))
        return _chunk("", B, rng.choice([hi, 1 + hi // 7, 1 + hi // 2]), hi, H, d, tau, fused, norm, fresh)
    if op == "step":
        return _step("", _log(rng, 1, 64), rng.choice([1, 5, 8, 16, 24, 32]), d, tau, fused, norm, fresh)
    if op == "norm":
        dn, H = rng.choice([8, 32, 64, 80, 96, 128, 128, 200, 256, 512]), rng.choice([1, 3, 8, 16, 32])
        return _norm("", _log(rng, 1, 50000000 // (H * dn)), H, dn, rng.choice([0, 1]), rng.choice([0, 1]), rng.choice([0, 1, 1]))
    B, Hq, Hk = _log(rng, 1, 64), rng.choice([1, 8, 16, 32]), rng.choice([0, 1, 4, 8])
    hi = _log(rng, 1, max(2, 1000000 // (B * (Hq + Hk))))
    return _rope("", B, rng.choice([hi, 1 + hi // 3]), hi, Hq, Hk, d, rng.choice([d, d, d // 2, 32]), rng.choice([0, 1]), rng.choice([0, 5000, 900000]),
                 rng.choice([10000.0, 640000.0, 5e6, 8e7]), rng.choice([1.0, 4.0]))


# ---- inputs -------------------------------------------------------------------------------------

def _lengths(case, seed):
    """Tokens of every sequence: the case fixes the set, the seed who has which."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    part = (np.arange(B) * 0.6180339887498949) % 1.0
    n = lo + np.round((hi - lo) * (1.0 - part / max(part.max(), 1e-9))).astype(np.int64)
    return n[np.random.RandomState(seed % (1 << 31)).permutation(B)].astype(np.int32)


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)


def prepare(case, seed):
    op, B, H, d = case["op"], case["B"], case["H"], case["d"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens = _lengths(case, seed)
    n = int(lens.sum())
    st = {"case": dict(case), "lens": lens}
    if op == "norm":
        xg = _normal(gen, n, 2 * H * d)
        st["x"], st["gate"] = _normal(gen, n, H * d) * 3 + 0.5, xg[:, H * d:] if case["gate"] else None
        st["gain"] = _normal(gen, H * d) * 0.2 + 1 if case["affine"] else None
        st["bias"] = _normal(gen, H * d) * 0.1 if case["affine"] else None
        st["y"] = torch.empty_like(st["x"])
    elif op == "rope":
        Hk, rot = case["Hk"], case["rot"]
        qk = _normal(gen, n, (H + Hk) * d)
        st["q"], st["k"] = qk[:, :H * d], qk[:, H * d:] if Hk else None
        st["freq"] = case["base"] ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot) / case["stretch"]
        r = np.random.RandomState((seed + 1) % (1 << 31))
        st["pos"] = (case["pos"] + r.randint(0, 1 + case["pos"] // 50, B)).astype(np.int32)
        st["qr"], st["kr"] = torch.empty_like(qk[:, :H * d]).contiguous(), torch.empty(n, Hk * d, dtype=torch.bfloat16, device="cuda") if Hk else None
        # every token's position (what a program with plain operations keeps beside its batch)
        st["at"] = torch.from_numpy(np.concatenate([p + np.arange(m) for p, m in zip(st["pos"], lens)])).cuda()
    else:
        if case["fused"]:                                          # slices of one projection: q, k, v, gate
            x = _normal(gen, n, 4 * H * d)
            st["q"], st["k"], st["v"], gate = (x[:, i * H * d:(i + 1) * H * d] for i in range(4))
        else:
            st["q"], st["k"], st["v"], gate = (_normal(gen, n, H * d) for _ in range(4))
        st["gate"] = gate if case["norm"] else None
        if case["tau"]:                                            # logits as the projection gives them
            st["decay"] = (torch.randn(n, H, generator=gen, device="cuda") * 1.5 + 1.0).to(torch.bfloat16)
        else:                                                      # fixed decays 1 - 2^-(2 .. 10) of the heads, a little apart from token to token
            rate = torch.log1p(-2.0 ** -(2.0 + 8.0 * torch.arange(H, device="cuda") / H))
            st["decay"] = rate * (0.5 + torch.rand(n, H, generator=gen, device="cuda"))
        # a pool of states: where every sequence's comes from (-1: it begins) and goes to
        r = np.random.RandomState((seed + 2) % (1 << 31))
        slots = r.permutation(2 * B + 1).astype(np.int32)
        st["from"], st["to"] = slots[:B].copy(), slots[B:2 * B].copy()
        if case["fresh"]:
            st["from"][::case["fresh"]] = -1
        st["state"] = torch.randn(2 * B + 1, H, d, d, generator=gen, device="cuda") * 3.0
        st["o"] = torch.empty(n, H * d, dtype=torch.bfloat16, device="cuda")
        first = np.concatenate([[0], np.cumsum(lens)])
        # places of the tokens in a padded batch, and back
        st["seq"] = torch.from_numpy(np.repeat(np.arange(B), lens)).cuda()
        st["in_seq"] = torch.from_numpy(np.arange(n) - np.repeat(first[:-1], lens)).cuda()
        st["from_dev"], st["to_dev"] = torch.from_numpy(st["from"].astype(np.int64)).cuda(), torch.from_numpy(st["to"].astype(np.int64)).cuda()
    if own:
        _plan(st)
    return st


# ---- the framework's calls ----------------------------------------------------------------------

def _plan(st):
    """The shapes, workspace and marshalled call that a serving loop keeps."""
    from paper_2405_05254_b200 import binding as yx
    c = st["case"]
    op, B, H, d, n = c["op"], c["B"], c["H"], c["d"], int(st["lens"].sum())
    if op == "norm":
        norm = yx.make_norm_gate(EPS, rms=c["rms"], gate=st["gate"], gain=st["gain"], bias=st["bias"])
        shape = yx.HeadNormShape(n, H, d, st["x"].stride(0), st["y"].stride(0))
        st["call"] = yx.prepare_tokens("yoco_head_norm", shape, st["x"], norm, st["y"])
    elif op == "rope":
        shape = yx.make_rope_shape(B, H, c["Hk"], d, c["hi"], rot=c["rot"], pairs=c["pairs"], q_stride=st["q"].stride(0),
                                   k_stride=st["k"].stride(0) if c["Hk"] else 0)
        st["call"] = yx.prepare_tokens("yoco_rope", shape, st["q"], st["k"], st["freq"], st["pos"], st["lens"], st["qr"], st["kr"])
    else:
        norm = yx.make_norm_gate(EPS, rms=c["norm"] == 2, gate=st["gate"]) if c["norm"] else None
        shape = yx.make_gret_shape(B, H, d, T=c["hi"], num_slots=2 * B + 1, tau=c["tau"], decay_bf16=bool(c["tau"]), q_stride=st["q"].stride(0),
                                   k_stride=st["k"].stride(0), v_stride=st["v"].stride(0))
        head = [shape, st["q"], st["k"], st["v"], st["decay"], norm, st["state"], st["from"], st["to"]]
        if op == "step":
            st["call"] = yx.prepare_tokens("yoco_gret_step", *head, st["o"])
        else:
            ws = torch.empty(yx.yoco_gret_workspace_size(shape, st["lens"]), dtype=torch.uint8, device="cuda")
            st["call"] = yx.prepare_tokens("yoco_gret_chunk", *head, st["lens"], st["o"], ws)


# ---- plain forms --------------------------------------------------------------------------------

def _norm_plain(x, rms, gate, gain, bias):
    """fp32 [n, H, d] -> fp32, normalised over d and gated."""
    if not rms:
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if gain is not None:
        x = x * gain.float().view(x.shape[1:]) + bias.float().view(x.shape[1:])
    if gate is not None:
        g = gate.float().reshape(x.shape)
        x = x * (g / (1.0 + torch.exp(-g)))
    return x


def _log_decay(st):
    """Natural logarithms of the decays, in 64 bits (sums of them run over long stretches)."""
    z = st["decay"].double()
    if not st["case"]["tau"]:
        return z
    return (torch.clamp(z, max=0.0) - torch.log1p(torch.exp(-z.abs()))) / st["case"]["tau"]


def _gret_out(st, o):
    """o: fp32 [n, H, d] of all tokens."""
    c = st["case"]
    if c["norm"]:
        o = _norm_plain(o, c["norm"] == 2, st["gate"], None, None)
    return {"O": o.to(torch.bfloat16).view(-1, c["H"] * c["d"]), "state": st["state"]}


def _first_states(st):
    s = st["state"][st["from_dev"].clamp(min=0)]
    return s * (st["from_dev"] >= 0).view(-1, 1, 1, 1)


def _step_plain(st):
    c = st["case"]
    B, H, d = c["B"], c["H"], c["d"]
    q, k, v = (st[x].float().reshape(B, H, d) for x in "qkv")
    s = _first_states(st) * torch.exp(_log_decay(st)).float()[..., None, None] + k[..., None] * v[..., None, :]
    st["state"][st["to_dev"]] = s
    return _gret_out(st, (q[:, :, None] @ s)[:, :, 0] * d ** -0.5)


def _chunk_plain(st):
    """In pieces of C tokens: inside a piece (q k^T * decays) v, from piece to piece the state."""
    c = st["case"]
    B, H, d, C = c["B"], c["H"], c["d"], 128
    top = int(st["lens"].max())
    C = min(C, top)
    N = -(-top // C)
    seq, at = st["seq"], st["in_seq"]

    def padded(x, width, dtype):                                   # [n, H * width] -> [B, N, H, C, width], zeros behind the sequences
        y = torch.zeros(B, N * C, H, width, dtype=dtype, device="cuda")
        y[seq, at] = x.to(dtype).reshape(-1, H, width)
        return y.view(B, N, C, H, width).transpose(2, 3)

    q, k, v = (padded(st[x], d, torch.float32) for x in "qkv")
    b = padded(_log_decay(st), 1, torch.float64)[..., 0].cumsum(-1)                       # [B, N, H, C]
    i = torch.arange(C, device="cuda")
    gap = torch.where(i[:, None] >= i, b[..., :, None] - b[..., None, :], torch.full((), -torch.inf, dtype=torch.float64, device="cuda"))
    o = ((q @ k.transpose(-1, -2)) * torch.exp(gap.float())) @ v
    del gap
    last = b[..., -1:]
    add = (k * torch.exp(last - b).float()[..., None]).transpose(-1, -2) @ v              # [B, N, H, d, d]
    keep = torch.exp(last).float()[..., None]
    s, before = _first_states(st), torch.empty_like(add)
    for n in range(N):
        before[:, n] = s
        s = s * keep[:, n] + add[:, n]
    o += (q * torch.exp(b).float()[..., None]) @ before
    st["state"][st["to_dev"]] = s
    return _gret_out(st, o.transpose(2, 3).reshape(B, N * C, H, d)[seq, at] * d ** -0.5)


def _rope_plain(st):
    c = st["case"]
    rot, d = c["rot"], c["d"]
    ang = st["at"].double()[:, None] * st["freq"]
    cos, sin = (torch.remainder(ang, 2 * np.pi).cos().float()[:, None], torch.remainder(ang, 2 * np.pi).sin().float()[:, None])
    out = {}
    for name, to in (("q", "qr"), ("k", "kr")):
        if st[name] is None:
            continue
        x = st[name].float().reshape(len(ang), -1, d)
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if c["pairs"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        a, b = a * cos - b * sin, b * cos + a * sin
        y = torch.stack((a, b), -1).flatten(-2) if c["pairs"] else torch.cat((a, b), -1)
        out[to] = torch.cat((y, x[..., rot:]), -1).to(torch.bfloat16).view(len(ang), -1)
    return out


def run(st):
    c = st["case"]
    op = c["op"]
    if own:
        st["call"].run()
        if op == "norm":
            return {"Y": st["y"]}
        if op == "rope":
            return {x: st[x] for x in ("qr", "kr") if st[x] is not None}
        return {"O": st["o"], "state": st["state"]}
    if op == "norm":
        x = _norm_plain(st["x"].float().view(-1, c["H"], c["d"]), c["rms"], st["gate"], st["gain"], st["bias"])
        return {"Y": x.to(torch.bfloat16).view(st["x"].shape)}
    return {"chunk": _chunk_plain, "step": _step_plain, "rope": _rope_plain}[op](st)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    op, B, H, d = case["op"], case["B"], case["H"], case["d"]
    lens = _lengths(case, 0)
    n = int(lens.sum())
    if op == "norm":
        return {"bytes": n * H * d * (6 if case["gate"] else 4) + case["affine"] * H * d * 4, "flops": n * H * d * 9}
    if op == "rope":
        return {"bytes": n * (H + case["Hk"]) * d * 4 + case["rot"] * 4, "flops": n * (H + case["Hk"]) * case["rot"] * 3}
    begin = -(-B // case["fresh"]) if case["fresh"] else 0
    moved = n * H * (8 * d + (2 * d if case["norm"] else 0) + (2 if case["tau"] else 4)) + (2 * B - begin) * H * d * d * 4
    return {"bytes": moved, "flops": n * H * 4 * d * d}                              # the recurrence: k^T v into S, q S


# ---- the definition in 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    op, B, H, d = case["op"], case["B"], case["H"], case["d"]

    def normalised(x, rms, gate, gain=None, bias=None):
        m = torch.zeros_like(x[..., :1]) if rms else x.sum(-1, keepdim=True) / d
        y = (x - m) / torch.sqrt(((x - m) ** 2).sum(-1, keepdim=True) / d + EPS)
        if gain is not None:
            y = gain.double().reshape(H, d) * y + bias.double().reshape(H, d)
        return y if gate is None else y * gate.double().reshape(y.shape) * torch.sigmoid(gate.double().reshape(y.shape))

    if op == "norm":
        return {"Y": normalised(st["x"].double().reshape(-1, H, d), case["rms"], st["gate"], st["gain"], st["bias"]).reshape(st["x"].shape)}
    if op == "rope":
        half, out = case["rot"] // 2, {}
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["at"].double()[:, None, None] * st["freq"])
        for name, to in (("q", "qr"), ("k", "kr")):
            if st[name] is None:
                continue
            y = st[name].double().reshape(len(st["at"]), -1, d).clone()
            first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["pairs"] else (slice(0, half), slice(half, 2 * half))
            z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
            y[..., first], y[..., second] = z.real, z.imag
            out[to] = y.reshape(len(st["at"]), -1)
        return out
    # the recurrence itself, all sequences a token at a time
    q, k, v = (st[x].double().reshape(-1, H, d) for x in "qkv")
    z = st["decay"].double()
    g = torch.sigmoid(z) ** (1.0 / case["tau"]) if case["tau"] else torch.exp(z)
    first = np.concatenate([[0], np.cumsum(st["lens"])])
    order = np.argsort(-st["lens"], kind="stable")                 # sequences that end first come last
    begin = torch.from_numpy(first[:-1][order]).cuda()
    s = torch.zeros(B, H, d, d, dtype=torch.float64, device="cuda")
    for i, b in enumerate(order):
        if st["from"][b] >= 0:
            s[i] = st["state"][int(st["from"][b])].double()
    o = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lens = st["lens"][order]
    for t in range(int(lens[0])):
        m = int((lens > t).sum())
        at = begin[:m] + t
        s[:m] = s[:m] * g[at][..., None, None] + k[at][..., None] * v[at][:, :, None]
        o[at] = (q[at][:, :, None] @ s[:m])[:, :, 0]
    state = st["state"].double()
    for i, b in enumerate(order):
        state[int(st["to"][b])] = s[i]
    o = o / d ** 0.5
    if case["norm"]:
        o = normalised(o, case["norm"] == 2, st["gate"])
    return {"O": o.reshape(-1, H * d), "state": state}
