"""The update with orthogonalised steps on matrices too large for one block, whose step is many launches: settings, gradients of any size, zeros,
what is not a number, and odd numbers of elements.  Bounds as oracle/muon.py derives them."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, sync
from test_gpu_muon import HYPER, check, matrix

pytestmark = pytest.mark.gpu
SHAPES = [(131, 301), (301, 131)]                     # both ways round, an element count that four does not divide


def launched(table):
    assert table.table.small == 0 and table.table.units[0][0] > 0
    return table


@pytest.mark.parametrize("kw", [dict(nesterov=0), dict(iterations=1), dict(iterations=2), dict(iterations=9), dict(momentum=0.0), dict(weight_decay=0.0),
                                dict(lr=0.0), dict(eps=1.0), dict(rms=0.0), dict(nesterov=0, iterations=4)], ids=str)
def test_settings(kw):
    kw = {k: float(np.float32(v)) if isinstance(v, float) else v for k, v in kw.items()}
    ms = [matrix(s, 5 + i, scale=0.01) for i, s in enumerate(SHAPES)]
    table = launched(mi.MuonTable(ms))
    table.workspace.fill_(0xFF)                                   # NaN wherever nothing was written
    for _ in range(2):
        check(ms, table, **kw)


@pytest.mark.parametrize("kw", [dict(nesterov=0, iterations=5), dict(iterations=2), dict(nesterov=0, iterations=4, momentum=0.0)], ids=str)
def test_settings_on_large_tiles(kw):
    shapes = [(513, 513), (300, 400), (700, 1300), (131, 301), (257, 300), (100, 401)] + 9 * [(2100, 520)]
    ms = [matrix(s, i) for i, s in enumerate(shapes)]
    table = launched(mi.MuonTable(ms))
    assert all(table.table.units[k][0] > 0 for k in range(7))
    table.workspace.fill_(0xFF)
    check(ms, table, **kw)


@pytest.mark.parametrize("scale", [1e-25, 1e-12, 1e18])
def test_gradients_of_any_size(scale):
    ms = [matrix(s, 1 + i, scale=scale) for i, s in enumerate(SHAPES)]
    check(ms, launched(mi.MuonTable(ms)), eps=1e-30)


@pytest.mark.parametrize("decay", [0.5, 2.0])
def test_singular_values_over_orders_of_magnitude(decay):
    ms = [matrix(s, 3 + i, decay=decay) for i, s in enumerate(SHAPES)]
    for t in ms:
        t["momentum"].zero_()
    check(ms, launched(mi.MuonTable(ms)))


def test_gradients_of_zeros():
    ms = [matrix(s, 7 + i) for i, s in enumerate(SHAPES)]
    for t in ms:
        t["grad"].zero_(), t["momentum"].zero_()
    before = [t["master"].clone() for t in ms]
    table = launched(mi.MuonTable(ms))
    for eps in (1e-7, 1e-30):
        mi.mimose_op_muon_step(table, lr=0.5, weight_decay=0.0, eps=eps)
    sync()
    for t, b in zip(ms, before):
        assert torch.equal(t["master"], b) and (t["momentum"] == 0).all()


@pytest.mark.parametrize("wrong", [float("nan"), float("inf")])
@pytest.mark.parametrize("parts", [1, 3])
def test_what_is_not_a_number_stays_in_its_matrix(parts, wrong):
    """Also where the next matrix works in the same scratch."""
    shapes = [(131, 301), (301, 131), (131, 301), (200, 260), (260, 200)]
    ms = [matrix(s, 9 + i) for i, s in enumerate(shapes)]
    alone = [{k: x.clone() for k, x in t.items()} for t in ms]
    ms[1]["grad"][3, 4] = wrong
    for _ in range(2):
        mi.mimose_op_muon_step(launched(mi.MuonTable(ms, parts=parts)), **HYPER)
        mi.mimose_op_muon_step(launched(mi.MuonTable(alone, parts=parts)), **HYPER)
    sync()
    assert not torch.isfinite(ms[1]["master"]).any()
    for i in (0, 2, 3, 4):
        assert torch.isfinite(ms[i]["master"]).all()
        assert all(torch.equal(ms[i][k], alone[i][k]) for k in ms[i])


@pytest.mark.parametrize("shape", [(8, 1024), (1024, 8), (1, 4096), (129, 129), (128, 257), (1024, 1024), (1024, 4096), (768, 130)])
def test_scratch_is_what_the_header_says(shape):
    table = mi.MuonTable([{k: torch.zeros(shape, device=DEV) for k in ("master", "grad", "momentum")} for _ in range(3)], parts=3)
    S, L = (-(-n // 128) * 128 for n in sorted(shape))
    assert table.table.parts == 3 and 4 * S * (S + L) < table.workspace.numel() <= 4 * S * (S + L) + 8192


def test_no_scratch_for_matrices_of_one_block():
    table = mi.MuonTable([{k: torch.zeros(s, device=DEV) for k in ("master", "grad", "momentum")} for s in ((128, 256), (256, 128), (3, 5))])
    assert table.workspace.numel() == 16


@pytest.mark.parametrize("rank", [1, 4, 17])
@pytest.mark.parametrize("shape", [(60, 140), (131, 301), (301, 131)], ids=str)
def test_gradients_of_low_rank(shape, rank):
    """The gradient of as few tokens: most singular values are 0 but for rounding, which the bound follows through the iterations."""
    t = matrix(shape, rank)
    g = torch.Generator().manual_seed(rank)
    u = torch.randn(shape[0], rank, generator=g, dtype=torch.float64) @ torch.randn(rank, shape[1], generator=g, dtype=torch.float64)
    t["grad"].copy_(u)
    t["momentum"].zero_()
    check([t], mi.MuonTable([t]))
