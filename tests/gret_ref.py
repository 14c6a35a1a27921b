"""Gated retention, head norm with gate and rotation from their definitions, in 64 bits on the CPU."""
import numpy as np


def log_decay(z, tau):
    """Natural logarithms of the decays."""
    z = np.asarray(z, dtype=np.float64)
    return (np.minimum(z, 0.0) - np.log1p(np.exp(-np.abs(z)))) / tau if tau else z


def retention(q, k, v, logs, lens, states, scale):
    """q, k, v [tokens, H, d], logs [tokens, H], states: list of [H, d, d] or None.  -> o, o_abs [tokens, H, d], states, states_abs.  The _abs forms
    are the same sums over magnitudes: what rounding errors are relative to."""
    _, H, d = q.shape
    o, o_abs = np.zeros(q.shape), np.zeros(q.shape)
    out, out_abs, t = [], [], 0
    for n, s0 in zip(lens, states):
        s = np.zeros((H, d, d)) if s0 is None else s0.astype(np.float64)
        a = np.abs(s)
        for _ in range(int(n)):
            g = np.exp(logs[t])[:, None, None]
            s = g * s + k[t][:, :, None] * v[t][:, None, :]
            a = g * a + np.abs(k[t])[:, :, None] * np.abs(v[t])[:, None, :]
            o[t] = scale * np.einsum("hk,hkv->hv", q[t], s)
            o_abs[t] = scale * np.einsum("hk,hkv->hv", np.abs(q[t]), a)
            t += 1
        out.append(s)
        out_abs.append(a)
    return o, o_abs, out, out_abs


def norm_gate(x, eps, rms, gate=None, gain=None, bias=None):
    """x [tokens, H, d] -> the same; gate as x, gain and bias [H, d]."""
    if not rms:
        x = x - x.mean(-1, keepdims=True)
    x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if gain is not None:
        x = x * gain
    if bias is not None:
        x = x + bias
    if gate is not None:
        with np.errstate(over="ignore"):
            x = x * gate / (1.0 + np.exp(-gate))
    return x


def rope(x, pos, freq, rot, pairs):
    """x [tokens, H, d] turned by the angles pos[token] * freq."""
    y = x.copy()
    ang = np.asarray(pos, dtype=np.float64)[:, None] * freq
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
