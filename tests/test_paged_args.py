"""Argument checks of the paged-cache entry points (host only: every refusal comes before anything is enqueued), and the
work plan of a paged call."""
import ctypes

import numpy as np
import pytest

from paper_2405_05254_b200 import binding as bd

vp = ctypes.c_void_p
A = vp(4096)                                   # an aligned address that is never followed


def lib():
    return bd.lib()


def layout(P=64, pages=100, stride=16, page_rows=0, cos=0, max_pos=0, pairs=0):
    return bd.PagedLayout(P, pages, stride, pairs, page_rows, cos or None, max_pos)


def host(a):
    arr = np.asarray(a, np.int32)
    return arr, vp(arr.ctypes.data)


def attend(fn="yoco_xattn_decode_paged", shape=None, lay=None, lens=(100, 1000), Q=A, K=A, V=A, s=A, table=A, O=A, lse=None, ws=A, size=0):
    """Default: a valid call but for its workspace, which is empty; without a device it cannot get further than that."""
    shape = shape or bd.make_shape(2, 8, 2, 128, 1)
    lay = lay or layout()
    keep, p = host(lens) if lens is not None else (None, None)
    pools = (K, s, V, s) if fn.endswith("_q4") else (K, V)
    return getattr(lib(), fn)(ctypes.byref(shape), ctypes.byref(lay), Q, *pools, table, p, O, lse, ws, size, None)


ATTEND = ["yoco_xattn_decode_paged", "yoco_xattn_decode_paged_q4", "yoco_xattn_chunk_paged", "yoco_xattn_chunk_paged_q4"]


@pytest.mark.parametrize("fn", ATTEND)
def test_attention_refuses_bad_arguments(fn):
    inv, uns = bd.ERR_INVALID_ARG, bd.ERR_UNSUPPORTED
    assert attend(fn) not in (bd.OK, inv, uns)                       # the base call is well formed
    for kw in ({"Q": None}, {"K": None}, {"V": None}, {"table": None}, {"O": None}, {"ws": None}, {"Q": vp(4100)},
               {"K": vp(4104)}, {"V": vp(4104)}, {"table": vp(4098)}, {"O": vp(4104)}, {"ws": vp(4096 + 128)}, {"lse": vp(4098)}):
        assert attend(fn, **kw) == inv, kw
    if fn.endswith("_q4"):
        assert attend(fn, s=None) == inv and attend(fn, s=vp(4104)) == inv
        assert attend(fn, shape=bd.make_shape(2, 8, 2, 64, 1)) == uns
    for P in (0, 1, 8, 24, 48, 512, -64):
        assert attend(fn, lay=layout(P=P, stride=4000)) == uns, P
    for lay in (layout(pages=0), layout(pages=-1), layout(stride=-1), layout(stride=15), layout(page_rows=127), layout(page_rows=-16),
                layout(pairs=2)):
        assert attend(fn, lay=lay) == inv
    assert attend(fn, lay=layout(page_rows=136)) == uns              # not a multiple of sixteen
    assert attend(fn, lay=layout(pages=2**31 // 128)) == uns         # row numbers pass 32 bits
    assert attend(fn, lay=layout(pages=2, page_rows=2**31)) == uns
    assert attend(fn, lens=(100, -1)) == inv
    assert attend(fn, lens=(100, 2**30 + 1), lay=layout(P=256, stride=2**23)) == uns
    assert attend(fn, lens=(100, 2**31 - 1), lay=layout(P=256, stride=2**23)) == uns
    assert attend(fn, lens=(100, 1025)) == inv                       # 17 pages in 16 entries
    assert attend(fn, shape=bd.make_shape(2, 8, 2, 128, 1, kv_head_stride=128 * 2000)) == inv
    assert attend(fn, shape=bd.make_shape(2, 7, 2, 128, 1)) == uns
    assert attend(fn, shape=bd.make_shape(2, 8, 2, 96, 1)) == uns
    assert attend(fn, shape=bd.make_shape(2, 8, 2, 128, 0)) == inv
    assert attend(fn, shape=bd.make_shape(2, 8, 2, 128, 1, scale=-1.0)) == inv
    assert attend(fn, shape=bd.make_shape(2, 8, 2, 128, 1, scale=float("nan"))) == inv
    assert attend(fn, lens=None, shape=bd.make_shape(2, 8, 2, 128, 1, max_kv_len=1025)) == inv
    assert getattr(lib(), fn)(None, None, *([A] * (9 if fn.endswith("_q4") else 7)), A, 0, None) == inv
    sh = bd.make_shape(2, 8, 2, 128, 1)
    assert getattr(lib(), fn)(ctypes.byref(sh), None, *([A] * (9 if fn.endswith("_q4") else 7)), A, 0, None) == inv
    assert attend(fn, shape=bd.make_shape(0, 8, 2, 128, 1), lens=()) == bd.OK
    if "decode" in fn:
        assert attend(fn, shape=bd.make_shape(2, 8, 2, 128, 5)) == uns   # 20 rows per KV head


def rows_call(fn, shape=None, lay=None, a=(3, 4), b=(100, 1000), src=A, pool=A, s=A, table=A, out=A):
    shape = shape or bd.PagedAppendShape(2, 2, 128, 1, 0)
    lay = lay or layout()
    ka, pa = host(a) if a is not None else (None, None)
    kb, pb = host(b) if b is not None else (None, None)
    pools = (pool, s, pool, s) if fn.endswith("_q4") else (pool, pool)
    if "append" in fn:
        return getattr(lib(), fn)(ctypes.byref(shape), ctypes.byref(lay), src, src, *pools, table, pa, pb, None)
    return getattr(lib(), fn)(ctypes.byref(shape), ctypes.byref(lay), *pools, table, pa, pb, out, out, None)


ROWS = ["yoco_paged_append", "yoco_paged_append_q4", "yoco_paged_gather", "yoco_paged_gather_q4"]


@pytest.mark.parametrize("fn", ROWS)
def test_append_and_gather_refuse_bad_arguments(fn):
    inv, uns = bd.ERR_INVALID_ARG, bd.ERR_UNSUPPORTED
    S = bd.PagedAppendShape
    for kw in ({"pool": None}, {"pool": vp(4104)}, {"table": None}, {"table": vp(4097)}, {"b": None}, {"b": (100, 1025)}, {"b": (100, -1)},
               {"a": (101, 4)}, {"a": (-1, 4)}):
        if "gather" in fn or kw != {"a": (101, 4)}:
            assert rows_call(fn, **kw) == inv, kw
    if "append" in fn:
        assert rows_call(fn, a=(101, 4)) == inv                       # more new tokens than the sequence has
        for kw in ({"src": None}, {"src": vp(4104)}, {"shape": S(2, 2, 128, 1, 255)}, {"shape": S(2, 2, 128, 1, -8)},
                   {"shape": S(2, 2, 128, -1, 0)}, {"a": None, "shape": S(2, 2, 128, 101, 0)}):
            assert rows_call(fn, **kw) == inv, kw
        assert rows_call(fn, shape=S(2, 2, 128, 1, 260)) == uns
        cos = 1 << 16
        assert rows_call(fn, lay=layout(cos=cos, max_pos=999)) == inv  # a position behind the table
        assert rows_call(fn, lay=layout(cos=cos + 8, max_pos=1000)) == inv
    else:
        assert rows_call(fn, out=None) == inv and rows_call(fn, out=vp(4104)) == inv and rows_call(fn, a=None) == inv
    if fn.endswith("_q4"):
        assert rows_call(fn, s=None) == inv and rows_call(fn, s=vp(4104)) == inv
        assert rows_call(fn, shape=S(2, 2, 64, 1, 0)) == uns
    assert rows_call(fn, a=(1, 1) if "append" in fn else (0, 0), b=(100, 2**30 + 1), lay=layout(P=256, stride=2**23)) == uns
    assert rows_call(fn, a=(2**29, 2**30) if "append" in fn else (2**29, 0), b=(2**30, 2**30), lay=layout(P=256, stride=2**23)) == uns
    for d in (0, 32, 96, 256):
        assert rows_call(fn, shape=S(2, 2, d, 1, 0)) == (inv if d == 0 else uns)
    assert rows_call(fn, shape=S(513, 2, 128, 1, 0)) == uns
    assert rows_call(fn, shape=S(-1, 2, 128, 1, 0)) == inv and rows_call(fn, shape=S(2, 0, 128, 1, 0)) == inv
    assert rows_call(fn, lay=layout(P=20)) == uns and rows_call(fn, lay=layout(page_rows=64)) == inv
    # nothing to do is no error and needs no device
    assert rows_call(fn, shape=S(0, 2, 128, 1, 0)) == bd.OK
    assert rows_call(fn, a=(0, 0) if "append" in fn else (100, 1000)) == bd.OK


def test_rope_q_refuses_bad_arguments():
    inv = bd.ERR_INVALID_ARG
    cos = 1 << 16

    def call(shape=None, lay=None, Q=A, lens=(100, 1000), R=A):
        shape = shape or bd.make_shape(2, 8, 2, 128, 1)
        lay = lay or layout(cos=cos, max_pos=1000)
        keep, p = host(lens)
        return lib().yoco_rope_q(ctypes.byref(shape), ctypes.byref(lay), Q, p, R, None)

    assert call(Q=None) == inv and call(R=None) == inv and call(Q=vp(4104)) == inv
    assert call(lay=layout()) == inv                                   # no table
    assert call(lay=layout(cos=cos, max_pos=999)) == inv
    assert call(lay=layout(cos=cos, max_pos=1000, pairs=3)) == inv
    assert call(lens=(100, -1)) == inv
    assert call(shape=bd.make_shape(2, 8, 2, 96, 1)) == bd.ERR_UNSUPPORTED
    assert call(shape=bd.make_shape(513, 8, 2, 128, 1), lens=[1] * 513) == bd.ERR_UNSUPPORTED
    assert call(shape=bd.make_shape(0, 8, 2, 128, 1), lens=[]) == bd.OK


def test_bad_page_status_word_and_error_texts():
    assert bd.yoco_xattn_decode_status_word(bd.STATUS_BAD_PAGE | (6 << 8)) == (bd.ERR_BAD_PAGE, bd.STATUS_BAD_PAGE, 5)
    texts = {lib().yoco_xattn_strerror(c) for c in range(-8, 1)}
    assert len(texts) == 9 and b"unknown error code" not in texts


def size(shape, lay, lens, mode, q4, sm=148):
    keep, p = host(lens)
    out = ctypes.c_size_t(0)
    rc = lib().yoco_xattn_workspace_size_paged(ctypes.byref(shape), ctypes.byref(lay), p, sm, mode, q4, ctypes.byref(out))
    return rc, out.value


def test_workspace_of_a_paged_call_is_that_of_the_packed_one():
    """The bf16 plan is the packed one; sequences may hold more keys than a packed cache could number (shared pages)."""
    for lens, T, mode in (([700, 3], 1, bd.MODE_DECODE), ([40000], 4, bd.MODE_DECODE), ([5000, 900], 300, bd.MODE_CHUNK)):
        sh = bd.make_shape(len(lens), 8, 2, 128, T)
        assert size(sh, layout(), lens, mode, 0) == (bd.OK, bd.yoco_xattn_workspace_size(sh, lens, mode, 148))
    lens = [1 << 20] * 300
    sh = bd.make_shape(300, 32, 8, 128, 1)
    keep, p = host(lens)
    out = ctypes.c_size_t(0)
    assert lib().yoco_xattn_workspace_size(ctypes.byref(sh), p, 148, bd.MODE_DECODE, ctypes.byref(out)) == bd.ERR_UNSUPPORTED
    assert size(sh, layout(), lens, bd.MODE_DECODE, 0)[0] == bd.OK
    assert size(sh, layout(P=48), lens, bd.MODE_DECODE, 0)[0] == bd.ERR_UNSUPPORTED
    assert size(bd.make_shape(1, 8, 2, 64, 1), layout(), [5], bd.MODE_DECODE, 1)[0] == bd.ERR_UNSUPPORTED


def test_the_binding_checks_tensors_before_the_call():
    """Host tensors, wrong types and short buffers are refused in Python, where a wrong address would reach the device."""
    import torch
    if not torch.cuda.is_available():
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            t = torch.zeros(8, dtype=torch.bfloat16)
            bd.prepare_paged("yoco_rope_q", bd.make_shape(1, 1, 1, 64, 1), layout(), t, [1], t)
    with pytest.raises(TypeError):
        bd.prepare_paged("yoco_rope_q", bd.make_shape(1, 1, 1, 64, 1), layout())
    with pytest.raises(ValueError):
        bd.make_paged_layout(16, 1, 1, cos_sin=torch.zeros(4, 128, dtype=torch.float64))


def test_the_binding_checks_strides():
    """What a call goes by is the base address and its row distances; a tensor that lies otherwise is refused."""
    import torch
    order = bd.PreparedPagedCall._in_order
    lay, wide = layout(P=16, pages=5, stride=7), layout(P=16, pages=5, stride=7, page_rows=2 * 3 * 16)
    new = bd.PagedAppendShape(2, 3, 64, 1, 0)
    fused = torch.zeros(9, 3 * 3 * 64)                                     # K, V and something else of every token
    slices = bd.PagedAppendShape(2, 3, 64, 1, 9 * 64)
    assert order("x", fused[:, :192], slices, lay) and order("x", fused[:, 192:384], slices, lay)
    assert order("x", fused.view(9, 9, 64)[:, 3:6], slices, lay) and order("x", fused.view(3, 3, 9, 64)[:, :, 3:6], slices, lay)
    assert not order("x", fused[:, :192], new, lay)                        # its tokens are not 192 elements apart
    assert not order("x", fused.t(), slices, lay) and not order("x", fused[::2, :192], slices, lay)
    assert not order("x", fused[:1, :192].expand(9, -1), slices, lay)
    assert order("x", torch.zeros(9, 192), new, lay) and order("x", torch.zeros(9 * 192), new, lay)
    assert order("x", fused[:1, :192], new, lay)                           # a single token has no distance
    pool = torch.zeros(5, 2, 3, 16, 64)
    assert order("k", pool[:, 0], new, wide) and order("k", pool[:, 1], new, wide) and order("k", pool, new, wide)
    assert not order("k", pool[:, 1], new, lay) and not order("k", pool.transpose(2, 3)[:, 0], new, wide)
    assert order("c", torch.zeros(5, 2, 3, 16, 32)[:, 1], new, wide) and order("s", torch.zeros(5, 2, 3, 16, 2)[:, 1], new, wide)
    assert order("k", torch.zeros(5, 3, 16, 64), new, lay)
    table = torch.zeros(2, 7, dtype=torch.int32)
    assert order("i", table, new, lay) and order("i", table.view(-1), new, lay) and order("i", table[:, :4], new, lay)
    assert not order("i", torch.zeros(2, 8, dtype=torch.int32), new, lay)
    assert not order("i", torch.zeros(7, 2, dtype=torch.int32).t(), new, lay)
    assert not order("q", torch.zeros(4, 4).t(), new, lay)
