"""The paged entry points on the host: refusals of the self-test of the bounded waits."""
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
