"""Sides of matrices that 32 bits do not hold: the library sees a side that it refuses, not what is left of it.  No GPU."""
import pytest

import paper_2209_02478_amd as mi
from test_muon_table_host import Tensor


def entry(shape):
    t = {name: Tensor(*shape) for name in ("master", "grad", "momentum")}
    for i, x in enumerate(t.values()):
        x.data_ptr = lambda at=1 << 40 + i: at
    return t


@pytest.mark.parametrize("shape", [((1 << 32) + 10, 1), (1, (1 << 32) + 10), ((1 << 32), 3), ((1 << 31) + 5, 1), ((1 << 20) + 1, 1)])
def test_sides(shape):
    with pytest.raises(mi.MimoseError, match="side"):
        mi.MuonTable([entry(shape)], stream=7)
