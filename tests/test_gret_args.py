"""Argument checks of retention, head norm and rotation (host only: every refusal comes before anything is enqueued)."""
import ctypes

import numpy as np
import pytest

from paper_2405_05254_b200 import binding as bd

vp = ctypes.c_void_p
A = vp(4096)                                   # an aligned address that is never followed
INV, UNS = bd.ERR_INVALID_ARG, bd.ERR_UNSUPPORTED


def host(a):
    if a is None:
        return None, None
    arr = np.asarray(a, np.int32)
    return arr, vp(arr.ctypes.data)


def gret(fn="yoco_gret_chunk", shape=None, Q=A, K=A, V=A, decay=A, norm=None, state=A, si=None, so=None, lens=(5, 300), O=A, ws=None, size=0, **kw):
    """Default: a valid call but for the device, without which it cannot get further."""
    s = shape or bd.make_gret_shape(2, 3, 128, T=5, num_slots=8, **kw)
    k1, p1 = host(si)
    k2, p2 = host(so)
    k3, p3 = host(lens)
    n = None if norm is None else ctypes.byref(norm)
    tail = (p3, O, ws, size, None) if fn == "yoco_gret_chunk" else (O, None)
    return getattr(bd.lib(), fn)(ctypes.byref(s), Q, K, V, decay, n, state, p1, p2, *tail)


BOTH = pytest.mark.parametrize("fn", ["yoco_gret_chunk", "yoco_gret_step"])


@BOTH
def test_retention_refuses_bad_arguments(fn):
    assert gret(fn) not in (bd.OK, INV, UNS)
    for kw in ({"Q": None}, {"K": None}, {"V": None}, {"decay": None}, {"state": None}, {"O": None}, {"Q": vp(4104)}, {"K": vp(4104)}, {"V": vp(4104)},
               {"O": vp(4104)}, {"state": vp(4104)}, {"decay": vp(4098)}, {"q_stride": 383}, {"q_stride": -8}, {"k_stride": 8}, {"v_stride": 376},
               {"o_stride": 376}, {"decay_stride": 2}, {"decay_stride": -1}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"tau": -1.0},
               {"tau": float("nan")}, {"tau": float("inf")}, {"tau": 1e-39}):
        assert gret(fn, **kw) == INV, kw
    for kw in ({"q_stride": 388}, {"k_stride": 388}, {"v_stride": 388}, {"o_stride": 388}):
        assert gret(fn, **kw) == UNS, kw
    mk = bd.make_gret_shape
    for s, rc in ((mk(-1, 3, 128, num_slots=8), INV), (mk(2, 0, 128, num_slots=8), INV), (mk(2, 3, 0, num_slots=8), INV), (mk(2, 3, 96, num_slots=8), UNS),
                  (mk(2, 3, 256, num_slots=8), UNS), (mk(513, 3, 128, num_slots=600), UNS), (mk(2, 65536, 128, num_slots=8), UNS), (mk(2, 3, 128, num_slots=-1), INV)):
        assert gret(fn, shape=s, lens=[1] * max(s.B, 1)) == rc, (s.B, s.H, s.d)
    bad = mk(2, 3, 128, num_slots=8)
    bad.decay_bf16 = 2
    assert gret(fn, shape=bad) == INV
    bf = mk(2, 3, 128, num_slots=8, decay_bf16=True)
    assert gret(fn, shape=bf, decay=vp(4098)) not in (INV, UNS) and gret(fn, shape=bf, decay=vp(4097)) == INV
    assert gret(fn, shape=mk(0, 3, 128, num_slots=8), lens=()) == bd.OK
    none = getattr(bd.lib(), fn)
    assert none(None, *([None] * (11 if fn.endswith("chunk") else 10)), *((0, None) if fn.endswith("chunk") else ())) == INV


@BOTH
def test_slots(fn):
    ok = gret(fn)
    for si, so, rc in (((0, 8), None, INV), ((0, -2), None, INV), (None, (0, 8), INV), (None, (-2, 1), INV), (None, (3, 3), INV), ((3, 3), (4, 5), ok),
                       ((3, 4), (4, 5), INV), ((3, 4), (3, 4), ok), ((3, 4), (4, 3), INV), ((-1, -1), (7, 6), ok), ((5, 5), (5, 6), INV), ((5, 5), (-1, -1), ok),
                       ((5, 6), (-1, 5), INV), ((5, 5), (-1, 5), INV)):
        assert gret(fn, si=si, so=so) == rc, (si, so)
    small = bd.make_gret_shape(2, 3, 128, num_slots=1)
    assert gret(fn, shape=small) == INV                       # slot 1 of one
    assert gret(fn, shape=small, si=(0, 0), so=(-1, -1)) == ok


@BOTH
def test_norm_and_gate(fn):
    ok = gret(fn)
    N = bd.NormGate
    assert gret(fn, norm=N(4096, None, None, 0, 1e-5, 0)) == ok and gret(fn, norm=N(None, None, None, 0, 0.0, 1)) == ok
    for n, rc in ((N(4104, None, None, 0, 1e-5, 0), INV), (N(4096, None, None, 100, 1e-5, 0), INV), (N(4096, None, None, 388, 1e-5, 0), UNS),
                  (N(4096, None, None, -8, 1e-5, 0), INV), (N(4096, 4100, None, 0, 1e-5, 0), INV), (N(4096, None, 4100, 0, 1e-5, 0), INV),
                  (N(4096, None, None, 0, -1.0, 0), INV), (N(4096, None, None, 0, float("nan"), 0), INV), (N(4096, None, None, 0, float("inf"), 0), INV),
                  (N(4096, None, None, 0, 1e-5, 2), INV)):
        assert gret(fn, norm=n) == rc


def test_lengths_and_workspace():
    assert gret(lens=(5, -1)) == INV and gret(lens=None, shape=bd.make_gret_shape(2, 3, 128, T=-1, num_slots=8)) == INV
    assert gret(lens=(2 ** 30, 1)) == UNS
    nothing = dict(lens=(0, 0), Q=None, K=None, V=None, decay=None, O=None)
    assert gret(**nothing) not in (INV, UNS)                  # states may still have to be handed on
    s = bd.make_gret_shape(2, 32, 128, num_slots=8)
    size = lambda shape, lens, sm: bd.yoco_gret_workspace_size(shape, lens, sm)  # noqa: E731
    assert size(s, [24, 3], 148) == 0 and size(s, [0, 0], 148) == 0 and size(bd.make_gret_shape(0, 32, 128), [], 148) == 0
    one = bd.make_gret_shape(1, 32, 128)
    assert size(one, [32768], 148) == 3 * 148 * (128 * 128 * 4 + 4)
    assert size(bd.make_gret_shape(1, 4, 64), [2560], 148) == 3 * 80 * (64 * 64 * 4 + 4)        # no more CTAs than chunks
    assert size(bd.make_gret_shape(8, 32, 128), [1000] * 8, 148) == 0                           # whole streams fill the device
    assert size(bd.make_gret_shape(1, 1, 128), [100], 148) == 0                                 # one chunk
    with pytest.raises(bd.YocoError):
        size(one, [-1], 148)
    with pytest.raises(bd.YocoError):
        size(bd.make_gret_shape(1, 32, 100), [5], 148)
    L = bd.lib()
    out = ctypes.c_size_t(0)
    assert L.yoco_gret_workspace_size(None, None, 148, ctypes.byref(out)) == INV
    assert L.yoco_gret_workspace_size(ctypes.addressof(one), None, 148, None) == INV


def norm_call(n=10, H=3, d=128, xs=0, ys=0, X=A, Y=A, norm=None):
    s = bd.HeadNormShape(n, H, d, xs, ys)
    ng = norm or bd.NormGate(None, None, None, 0, 1e-5, 0)
    return bd.lib().yoco_head_norm(ctypes.addressof(s), X, ctypes.addressof(ng), Y, None)


def test_head_norm_refuses_bad_arguments():
    assert norm_call() not in (bd.OK, INV, UNS)
    for kw in ({"n": -1}, {"H": 0}, {"d": 0}, {"d": -8}, {"xs": -8}, {"ys": 376}, {"xs": 376}, {"X": None}, {"Y": None}, {"X": vp(4104)}, {"Y": vp(4104)},
               {"norm": bd.NormGate(4104, None, None, 0, 1e-5, 0)}, {"norm": bd.NormGate(None, None, None, 0, -1e-5, 0)}):
        assert norm_call(**kw) == INV, kw
    for kw in ({"d": 12}, {"d": 1032}, {"xs": 388}, {"ys": 388}, {"n": 2 ** 30}, {"n": 2 ** 62}):
        assert norm_call(**kw) == UNS, kw
    assert norm_call(n=0, X=None, Y=None) == bd.OK
    s = bd.HeadNormShape(10, 3, 128, 0, 0)
    assert bd.lib().yoco_head_norm(None, A, A, A, None) == INV and bd.lib().yoco_head_norm(ctypes.addressof(s), A, None, A, None) == INV


def rope_call(shape=None, Q=A, K=A, freq=A, pos=(0, 5), lens=(3, 4), Qr=A, Kr=A, **kw):
    s = shape or bd.make_rope_shape(2, 4, 2, 128, T=1, **kw)
    k1, p1 = host(pos)
    k2, p2 = host(lens)
    return bd.lib().yoco_rope(ctypes.addressof(s), Q, K, freq, p1, p2, Qr, Kr, None)


def test_rotation_refuses_bad_arguments():
    mk = bd.make_rope_shape
    assert rope_call() not in (bd.OK, INV, UNS)
    for kw in ({"Q": None}, {"K": None}, {"Qr": None}, {"Kr": None}, {"freq": None}, {"freq": vp(4100)}, {"pos": None}, {"pos": (0, -1)}, {"lens": (3, -1)},
               {"Q": vp(4104)}, {"K": vp(4104)}, {"Qr": vp(4104)}, {"Kr": vp(4104)}, {"q_stride": 504}, {"k_stride": 248}, {"q_out_stride": 8},
               {"k_out_stride": -8}, {"rot": 144}, {"rot": -16}, {"pairs": 2}, {"pos": (0, 2 ** 31 - 3)}):
        assert rope_call(**kw) == INV, kw
    for kw in ({"rot": 24}, {"q_stride": 516}, {"k_out_stride": 260}, {"lens": (2 ** 30, 1)}, {"shape": mk(2, 4, 2, 100)}, {"shape": mk(2, 4, 2, 528)},
               {"shape": mk(513, 4, 2, 128)}, {"shape": mk(2, 65535, 1, 16)}):
        if "shape" in kw:
            kw = dict(kw, pos=[0] * kw["shape"].B, lens=[1] * kw["shape"].B)
        assert rope_call(**kw) == UNS, kw
    for s in (mk(-1, 4, 2, 128), mk(2, 0, 2, 128), mk(2, 4, -1, 128), mk(2, 4, 2, 0)):
        assert rope_call(shape=s) == INV
    assert rope_call(shape=mk(0, 4, 2, 128), pos=(), lens=()) == bd.OK
    assert rope_call(lens=(0, 0), Q=None, K=None, Qr=None, Kr=None) == bd.OK
    assert rope_call(pos=(0, 2 ** 31 - 4)) not in (INV, UNS)                  # the last position there is
    assert rope_call(shape=mk(2, 4, 0, 128, T=1), K=None, Kr=None) not in (INV, UNS)
    assert bd.lib().yoco_rope(None, A, A, A, None, None, A, A, None) == INV


def test_in_place_needs_rows_of_one_distance():
    B = vp(1 << 20)
    ok = norm_call()
    assert norm_call(xs=392) == INV and norm_call(ys=392) == INV and norm_call(xs=392, ys=392) == ok and norm_call(xs=392, Y=B) == ok
    assert norm_call(n=1, xs=392) == ok
    ok = rope_call()
    assert rope_call(q_stride=520) == INV and rope_call(k_out_stride=264) == INV and rope_call(q_stride=520, q_out_stride=520) == ok
    assert rope_call(q_stride=520, Qr=B) == ok and rope_call(k_stride=264, Kr=B) == ok and rope_call(lens=(1, 0), q_stride=520) == ok


def test_structures_have_the_sizes_of_the_header():
    assert ctypes.sizeof(bd.GretShape) == 72 and ctypes.sizeof(bd.NormGate) == 40 and ctypes.sizeof(bd.HeadNormShape) == 32
    assert ctypes.sizeof(bd.RopeShape) == 64
