"""Host side of gated retention: what the calls refuse beside their own arguments' ranges."""
import ctypes

import numpy as np
import pytest

from paper_2405_05254_b200 import binding as bd


def test_a_workspace_for_fewer_lengths_than_sequences_is_refused():
    shape = bd.make_gret_shape(4, 32, 128)
    for lens in ([], [300], [300, 5, 7]):
        with pytest.raises(ValueError):
            bd.yoco_gret_workspace_size(shape, lens, 148)
    assert bd.yoco_gret_workspace_size(shape, [300, 5, 7, 0], 148) == bd.yoco_gret_workspace_size(shape, [300, 5, 7, 0, 9], 148)
    with pytest.raises(ValueError):
        bd.yoco_gret_workspace_bound(shape, [300], 148)


@pytest.mark.parametrize("H,d", [(1, 128), (5, 64), (32, 128), (37, 64)])
def test_a_workspace_for_lengths_up_to_those_given(H, d):
    """The exact size is not monotone: a few streams are cut where many are dealt out whole."""
    r = np.random.RandomState(H)
    for lens in ([1000] * 8, [4096] * 5, [100], [18] * 4, [19, 1], [2600, 777, 3, 1900], [130] * 30, r.randint(0, 5000, 12), [70000, 3]):
        lens = np.asarray(lens, np.int32)
        shape = bd.make_gret_shape(len(lens), H, d)
        bound = bd.yoco_gret_workspace_bound(shape, lens, 148)
        assert bound <= 3 * 148 * (d * d + 1) * 4
        for _ in range(60):
            now = np.where(r.rand(len(lens)) < r.rand(), 0, (lens * r.rand(len(lens)) ** r.choice([0.0, 0.3, 2.0])).astype(np.int32))
            assert bd.yoco_gret_workspace_size(shape, now, 148) <= bound, (lens, now)
            assert bd.yoco_gret_workspace_bound(shape, now, 148) <= bound
    eight, one = [1000] * 8, [1000] + [0] * 7
    shape = bd.make_gret_shape(8, 32, 128, T=1000)
    assert bd.yoco_gret_workspace_size(shape, eight, 148) == 0 < bd.yoco_gret_workspace_size(shape, one, 148) <= bd.yoco_gret_workspace_bound(shape, eight, 148)
    assert bd.yoco_gret_workspace_bound(shape, None, 148) == bd.yoco_gret_workspace_bound(shape, eight, 148)
    assert bd.yoco_gret_workspace_bound(shape, [18] * 8, 148) == 0
    for bad in (bd.make_gret_shape(1, 32, 100), bd.make_gret_shape(1, 32, 128, T=-1)):
        with pytest.raises(bd.YocoError):
            bd.yoco_gret_workspace_bound(bad, None, 148)


def test_the_self_test_of_the_waits_checks_its_arguments():
    A = ctypes.c_void_p(4096)
    L = bd.lib()
    shape = bd.make_gret_shape(1, 2, 128, T=300)

    def call(limit_ms, Q=A):
        return L.yoco_gret_selftest_wait_expiry(ctypes.addressof(shape), Q, A, A, A, None, A, None, None, None, A, None, 0, limit_ms, None)

    for ms in (0, -1, 1001):
        assert call(ms) == bd.ERR_INVALID_ARG
    assert call(20, Q=None) == bd.ERR_INVALID_ARG and call(20) not in (bd.OK, bd.ERR_INVALID_ARG, bd.ERR_UNSUPPORTED)
