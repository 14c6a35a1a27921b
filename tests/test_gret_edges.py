"""Host side of gated retention: what the calls refuse beside their own arguments' ranges."""
import pytest

from paper_2405_05254_b200 import binding as bd


def test_a_workspace_for_fewer_lengths_than_sequences_is_refused():
    shape = bd.make_gret_shape(4, 32, 128)
    for lens in ([], [300], [300, 5, 7]):
        with pytest.raises(ValueError):
            bd.yoco_gret_workspace_size(shape, lens, 148)
    assert bd.yoco_gret_workspace_size(shape, [300, 5, 7, 0], 148) == bd.yoco_gret_workspace_size(shape, [300, 5, 7, 0, 9], 148)
