"""The paged entry points on the host: refusals of the self-test of the bounded waits, workspaces of growing sequences."""
import ctypes

import numpy as np
import pytest

from paper_2405_05254_b200 import binding as bd
from test_paged_args import A, host, layout, lib, vp


def test_the_self_test_of_the_waits_refuses_bad_arguments():
    sh, lay = bd.make_shape(2, 8, 2, 128, 1), layout()
    keep, p = host((100, 1000))

    def call(shape=sh, K=A, Ks=A, Vs=A, O=A, ws=A, ms=20):
        return lib().yoco_xattn_selftest_wait_expiry_paged(ctypes.byref(shape), ctypes.byref(lay), A, K, Ks, A, Vs, A, p, O, ws, 0, ms, None)

    inv = bd.ERR_INVALID_ARG
    assert call() not in (bd.OK, inv, bd.ERR_UNSUPPORTED) and call(Ks=None, Vs=None) not in (bd.OK, inv, bd.ERR_UNSUPPORTED)
    for kw in ({"ms": 0}, {"ms": 1001}, {"ms": -5}, {"Ks": None}, {"Vs": None}, {"K": None}, {"O": None}, {"ws": None}, {"Ks": vp(4104)}):
        assert call(**kw) == inv, kw
    assert call(shape=bd.make_shape(2, 8, 2, 64, 1)) == bd.ERR_UNSUPPORTED
    assert call(shape=bd.make_shape(2, 8, 2, 128, 5)) == bd.ERR_UNSUPPORTED


def workspace(fn, shape, lens, mode, q4, sm=148):
    keep, p = host(lens)
    out = ctypes.c_size_t(0)
    rc = getattr(lib(), fn)(ctypes.byref(shape), ctypes.byref(layout()), p, sm, mode, q4, ctypes.byref(out))
    assert rc == bd.OK
    return out.value


SIZE, BOUND = "yoco_xattn_workspace_size_paged", "yoco_xattn_workspace_bound_paged"


def test_the_exact_workspace_of_shorter_sequences_can_be_the_larger_one():
    """Why the bound is needed: sequences that grow within a workspace sized for their last lengths."""
    sh = bd.make_shape(16, 32, 8, 128, 1)
    assert workspace(SIZE, sh, [2560] * 16, bd.MODE_DECODE, 1) > workspace(SIZE, sh, [2688] * 16, bd.MODE_DECODE, 1)
    assert workspace(BOUND, sh, [2688] * 16, bd.MODE_DECODE, 1) >= workspace(SIZE, sh, [2560] * 16, bd.MODE_DECODE, 1)


@pytest.mark.parametrize("q4", [0, 1])
@pytest.mark.parametrize("mode,T,window", [(bd.MODE_DECODE, 1, 0), (bd.MODE_DECODE, 4, 0), (bd.MODE_DECODE, 2, 100), (bd.MODE_DECODE, 1, 1),
                                           (bd.MODE_CHUNK, 9, 0), (bd.MODE_CHUNK, 300, 0), (bd.MODE_CHUNK, 40, 1000),
                                           (bd.MODE_DECODE, 1, 2**31 - 1)])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 32, 8), (3, 4, 1), (16, 32, 8), (64, 8, 2), (90, 32, 8)])
def test_the_workspace_bound_covers_every_length_up_to_the_given_ones(q4, mode, T, window, B, Hq, Hkv):
    r = np.random.default_rng(B * 31 + T)
    sh = bd.make_shape(B, Hq, Hkv, 128, T, window=window)
    for longest in (50, 1537, 2752, 6000, 70000, 300000 if B < 20 else 9000):
        tops = [np.full(B, longest), r.integers(0, longest + 1, B)]
        for top in tops:
            bound = workspace(BOUND, sh, top, mode, q4)
            assert bound <= workspace(BOUND, sh, top + 64, mode, q4)              # it grows with the lengths
            tries = [top, top // 2, np.zeros(B, np.int64)] + [np.minimum(top, n) for n in r.integers(1, longest + 1, 12)]
            tries += [np.minimum(top, r.integers(0, longest + 1, B)) for _ in range(12)]
            tries += [np.minimum(top, np.where(r.random(B) < 0.3, longest, 64)) for _ in range(3)]
            for lens in tries:
                assert workspace(SIZE, sh, lens, mode, q4) <= bound, (lens, top)


@pytest.mark.parametrize("q4", [0, 1])
def test_the_workspace_bound_over_every_tile_of_a_growing_batch(q4):
    for B, Hkv, top in ((1, 8, 9000), (8, 8, 4200), (16, 8, 3000), (2, 2, 40000)):
        sh = bd.make_shape(B, 4 * Hkv, Hkv, 128, 1)
        bound = workspace(BOUND, sh, [top] * B, bd.MODE_DECODE, q4)
        for n in range(1, top + 1, 64):
            assert workspace(SIZE, sh, [n] * B, bd.MODE_DECODE, q4) <= bound, n


@pytest.mark.parametrize("sm", [1, 7, 132, 148])
def test_the_workspace_bound_where_groups_have_pieces(sm):
    """bf16 decode cuts long groups into two or four pieces, and not where groups are chains of short streams."""
    r = np.random.default_rng(sm)
    for B, Hkv in ((1, 1), (2, 8), (30, 8), (80, 8)):
        sh = bd.make_shape(B, 4 * Hkv, Hkv, 128, 1)
        for _ in range(20):
            top = r.integers(0, int(10 ** r.uniform(2, 5.5)) + 1, B)
            bound = workspace(BOUND, sh, top, bd.MODE_DECODE, 0, sm)
            for _ in range(10):
                lens = np.minimum(top, (top * r.random(B) ** r.integers(0, 4)).astype(np.int64))
                assert workspace(SIZE, sh, lens, bd.MODE_DECODE, 0, sm) <= bound


def test_the_workspace_bound_refuses_what_the_size_refuses():
    out = ctypes.c_size_t(0)
    keep, p = host((100, 1000))
    keep2, bad = host((100, -1))

    def call(shape=bd.make_shape(2, 8, 2, 128, 1), lay=layout(), lens=p, sm=148, mode=bd.MODE_DECODE, q4=0, o=ctypes.byref(out)):
        return lib().yoco_xattn_workspace_bound_paged(ctypes.byref(shape) if shape else None, ctypes.byref(lay) if lay else None, lens, sm, mode, q4, o)

    assert call() == bd.OK and out.value > 0
    for kw in ({"shape": None}, {"lay": None}, {"sm": -1}, {"mode": 2}, {"lens": bad}, {"o": None},
               {"shape": bd.make_shape(2, 8, 2, 128, 1, kv_head_stride=128 * 2000)}):
        assert call(**kw) == bd.ERR_INVALID_ARG, kw
    assert call(lay=layout(P=48)) == bd.ERR_UNSUPPORTED and call(shape=bd.make_shape(2, 8, 2, 64, 1), q4=1) == bd.ERR_UNSUPPORTED
    assert call(shape=bd.make_shape(2, 8, 2, 128, 5)) == bd.ERR_UNSUPPORTED


def test_the_binding_checks_the_strides_of_contiguous_tensors_too():
    """A contiguous tensor whose rows are wider than the call's would be read at the wrong distance."""
    import torch
    order = bd.PreparedPagedCall._in_order
    lay, wide = layout(P=16, pages=5, stride=7), layout(P=16, pages=5, stride=7, page_rows=2 * 3 * 16)
    new, fused = bd.PagedAppendShape(2, 3, 64, 1, 0), bd.PagedAppendShape(2, 3, 64, 1, 9 * 64)
    qkv = torch.zeros(9, 9 * 64)                                    # a projection's whole output
    assert not order("x", qkv, new, lay) and not order("x", qkv.view(9, 9, 64), new, lay)
    assert order("x", qkv, fused, lay) and order("x", qkv.view(9, 9, 64), fused, lay) and order("x", qkv.view(9, 3, 3, 64), fused, lay)
    assert order("x", qkv.view(9, 3, 192)[:, 1], fused, lay) and not order("x", qkv.view(9, 3, 192)[:, 1], new, lay)
    own = torch.zeros(9, 3 * 64)
    assert order("x", own, new, lay) and order("x", own.view(9, 3, 64), new, lay) and order("x", own.view(3, 3, 3, 64), new, lay)
    assert not order("x", own, fused, lay) and not order("x", own.view(9, 3, 64), fused, lay)   # its tokens are 192 apart
    assert order("x", own[:1], fused, lay)                          # a single token has no distance
    assert order("x", torch.zeros(0, 192), new, lay) and order("x", torch.zeros(0, 192), fused, lay)
    for kind, e in (("k", 64), ("c", 32), ("s", 2)):
        both, one = torch.zeros(5, 2, 3, 16, e), torch.zeros(5, 3, 16, e)
        assert order(kind, both, new, wide) and order(kind, one, new, lay)
        assert order(kind, torch.zeros(10, 3, 16, e), new, wide)                                         # K and V pages in turn
        assert not order(kind, torch.zeros(5, 4, 16, e), new, lay)                                       # pages of four heads
        assert not order(kind, torch.zeros(5, 3, 32, e), new, lay)                                       # ... of 32 tokens
        assert order(kind, one.view(-1, e), new, lay) and order(kind, one.view(-1), new, wide)           # flat: as the caller says
        assert order(kind, torch.zeros(8, 3, 16, e), new, lay)                                           # spare pages
    table = torch.zeros(2, 7, dtype=torch.int32)
    assert order("i", table, new, lay) and order("i", table.view(-1), new, lay)
    assert not order("i", torch.zeros(2, 8, dtype=torch.int32), new, lay) and not order("i", torch.zeros(4, 6, dtype=torch.int32), new, lay)
    assert order("i", torch.zeros(1, 8, dtype=torch.int32), new, lay)


@pytest.mark.parametrize("fn", ["yoco_paged_append", "yoco_paged_append_q4", "yoco_paged_gather", "yoco_paged_gather_q4"])
def test_calls_without_a_token_take_empty_tensors(fn):
    """An empty tensor's address is null: no token to store or read back is no error; with a token a null address is."""
    from test_paged_args import rows_call
    none = (0, 0) if "append" in fn else (100, 1000)
    assert rows_call(fn, a=none, src=None, out=None) == bd.OK
    if "append" in fn:
        assert rows_call(fn, a=None, shape=bd.PagedAppendShape(2, 2, 128, 0, 0), src=None) == bd.OK
        assert rows_call(fn, a=(0, 1), src=None) == bd.ERR_INVALID_ARG
    else:
        assert rows_call(fn, a=(100, 999), out=None) == bd.ERR_INVALID_ARG
    assert rows_call(fn, a=none, src=vp(4104), out=vp(4104)) == bd.ERR_INVALID_ARG
    assert rows_call(fn, a=none, src=None, out=None, pool=None) == bd.ERR_INVALID_ARG
