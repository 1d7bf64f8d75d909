"""The update with orthogonalised steps against its definition in 64 bits; bounds as oracle/muon.py derives them."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, sync
from oracle import muon as om

pytestmark = pytest.mark.gpu
HYPER = dict(lr=0.5, momentum=0.9, weight_decay=0.01, rms=0.2, eps=1e-7, nesterov=1, iterations=5)
HYPER = {k: float(np.float32(v)) if isinstance(v, float) else v for k, v in HYPER.items()}


def matrix(shape, seed, scale=1.0, decay=0.0, lowp=True, w=0.02):
    rng = np.random.default_rng(seed)
    g = rng.standard_normal(shape)
    if decay:
        U, s, V = np.linalg.svd(g, full_matrices=False)
        g = U * (1.0 / (1 + np.arange(len(s))) ** decay) @ V
    t = dict(grad=torch.tensor(g * scale, dtype=torch.float32, device=DEV), momentum=torch.tensor(rng.standard_normal(shape) * scale, dtype=torch.float32, device=DEV),
             master=torch.tensor(rng.standard_normal(shape) * w, dtype=torch.float32, device=DEV))
    if lowp:
        t["lowp"] = torch.zeros(shape, dtype=torch.bfloat16, device=DEV)
    return t


def values(t):
    return {k: x.double().cpu().numpy() for k, x in t.items()}


def check(matrices, table, **kw):
    h = HYPER | kw
    before = [values(t) for t in matrices]
    mi.mimose_op_muon_step(table, **h)
    sync()
    for t, b in zip(matrices, before):
        if t["master"].numel() == 0:
            continue
        w, m, off = om.step(b["master"], b["grad"], b["momentum"], **h)
        got = values(t)
        assert np.isfinite(got["master"]).all()
        m_off = 4 * om.F32 * (np.abs(h["momentum"] * b["momentum"]) + np.abs(b["grad"])) + 2.0 ** -149
        assert (np.abs(got["momentum"] - m) <= m_off).all(), b["master"].shape
        far = np.linalg.norm(got["master"] - w)
        assert far <= off, (b["master"].shape, far, off)
        assert (got["grad"] == b["grad"]).all()
        if "lowp" in t:
            assert torch.equal(t["lowp"], t["master"].bfloat16())


SHAPES = [(1, 1), (1, 9), (9, 1), (3, 4), (64, 64), (65, 130), (130, 65), (128, 128), (127, 129), (129, 257), (300, 77), (77, 300), (256, 256), (128, 256), (256, 128), (128, 257), (129, 256), (33, 200)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_one_matrix(shape):
    ms = [matrix(shape, sum(shape))]
    table = mi.MuonTable(ms)
    for _ in range(2):                                            # the second step starts from the first one's momentum
        check(ms, table)


def test_large_tiles():
    """Enough tiles of 256 to be used, whole and not, beside smaller ones; and the same bits without them, in more parts."""
    shapes = [(513, 513), (700, 1300), (64, 70), (1300, 700), (640, 520), (300, 400), (768, 768), (520, 2100), (130, 1000), (257, 300)] + 7 * [(2100, 520)]

    def fresh():
        return [matrix(s, i) for i, s in enumerate(shapes)]

    ms = fresh()
    table = mi.MuonTable(ms)
    assert table.table.parts == 1 and all(table.table.units[k][0] > 0 for k in range(7))
    table.workspace.fill_(0xFF)
    check(ms, table)
    others = fresh()
    several = mi.MuonTable(others, parts=6)
    assert not any(several.table.units[k][several.table.parts - 1] for k in (4, 5, 6))
    several.workspace.fill_(0xFF)
    mi.mimose_op_muon_step(several, **HYPER)
    sync()
    assert all(torch.equal(a["master"], b["master"]) for a, b in zip(ms, others))
    check(ms, table)


@pytest.mark.parametrize("parts", [1, 2, 5, 64])
def test_lists(parts):
    """Matrices of all shapes in one list, in as many parts as asked for and in scratch of that size."""
    ms = [matrix(s, i, lowp=i % 2 == 0) for i, s in enumerate(SHAPES + [(0, 5), (5, 0)])]
    table = mi.MuonTable(ms, parts=parts)
    assert 1 <= table.table.parts <= parts
    assert parts > 1 or table.table.parts == 1
    table.workspace.fill_(0xFF)                                   # NaN wherever nothing was written
    check(ms, table)
    whole = mi.MuonTable(ms).workspace.numel()
    assert table.workspace.numel() <= whole and (parts < 5 or table.workspace.numel() < whole // 2)


@pytest.mark.parametrize("scale", [1e-25, 1e-12, 1e18])
def test_gradients_of_any_size(scale):
    ms = [matrix((70, 130), 1, scale=scale), matrix((130, 70), 2, scale=scale)]
    check(ms, mi.MuonTable(ms), eps=1e-30)


@pytest.mark.parametrize("decay", [0.5, 1.0, 2.0])
def test_singular_values_over_orders_of_magnitude(decay):
    ms = [matrix((96, 200), 3, decay=decay), matrix((200, 200), 4, decay=decay)]
    for t in ms:
        t["momentum"].zero_()
    check(ms, mi.MuonTable(ms))


@pytest.mark.parametrize("kw", [dict(nesterov=0), dict(iterations=1), dict(iterations=2), dict(iterations=9), dict(momentum=0.0), dict(weight_decay=0.0),
                                dict(lr=0.0), dict(eps=1.0), dict(rms=0.0)], ids=str)
def test_settings(kw):
    kw = {k: float(np.float32(v)) if isinstance(v, float) else v for k, v in kw.items()}
    ms = [matrix((60, 140), 5, scale=0.01), matrix((140, 60), 6, scale=0.01)]
    check(ms, mi.MuonTable(ms), **kw)


def test_gradients_of_zeros():
    ms = [matrix((40, 50), 7), matrix((50, 40), 8)]
    for t in ms:
        t["grad"].zero_(), t["momentum"].zero_()
    before = [t["master"].clone() for t in ms]
    table = mi.MuonTable(ms)
    for eps in (1e-7, 1e-30):
        mi.mimose_op_muon_step(table, lr=0.5, weight_decay=0.0, eps=eps)
    sync()
    for t, b in zip(ms, before):
        assert torch.equal(t["master"], b) and (t["momentum"] == 0).all()


def test_what_is_not_a_number_stays_in_its_matrix():
    ms = [matrix((60, 60), 9), matrix((60, 60), 10), matrix((60, 60), 11)]
    alone = [{k: x.clone() for k, x in t.items()} for t in ms]
    ms[1]["grad"][3, 4] = float("nan")
    mi.mimose_op_muon_step(mi.MuonTable(ms), **HYPER)
    mi.mimose_op_muon_step(mi.MuonTable(alone), **HYPER)
    sync()
    assert torch.isnan(ms[1]["master"]).all()
    for i in (0, 2):
        assert torch.equal(ms[i]["master"], alone[i]["master"])


def test_the_same_whatever_the_list():
    """A matrix' result does not depend on what else is in the list, on its place or on the parts, and is the same each time."""
    def fresh():
        return [matrix(s, i) for i, s in enumerate([(200, 300), (64, 64), (300, 200)])]
    results = []
    for order, parts in (([0, 1, 2], 1), ([2, 0, 1], 1), ([0, 1, 2], 3), ([0, 1, 2], 1)):
        ms = fresh()
        mi.mimose_op_muon_step(mi.MuonTable([ms[i] for i in order], parts=parts), **HYPER)
        sync()
        results.append([t["master"] for t in ms])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))


def test_tiles_of_128_and_of_64():
    """Enough tiles of 128 to be used; and the same bits in parts that have too few and take those of 64."""
    shapes = 30 * [(383, 383)]
    results = []
    for parts in (1, 2, 8):
        ms = [matrix(s, i) for i, s in enumerate(shapes)]
        table = mi.MuonTable(ms, parts=parts)
        every = (1 << table.table.parts) - 1
        assert list(table.table.fine) == {1: [0, 0], 2: [every, 0], 8: [every, every]}[parts]
        if parts == 1:
            check(ms, table)
        else:
            mi.mimose_op_muon_step(table, **HYPER)
        sync()
        results.append([t[k] for t in ms for k in sorted(t)])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, results[0]))


def test_captured_on_two_workspaces():
    """Two captured steps with a workspace each, replayed side by side, beside an eager one."""
    sets = [[matrix((90, 150), s), matrix((310, 150), s + 1)] for s in (20, 30, 40)]
    eager = [[{k: x.clone() for k, x in t.items()} for t in ms] for ms in sets]
    tables = [mi.MuonTable(ms) for ms in sets]
    for table in tables:
        mi.mimose_op_muon_step(table, **(HYPER | dict(lr=0.0)))
    for ms, es in zip(sets, eager):
        for t, e in zip(ms, es):
            for k in t:
                t[k].copy_(e[k])
    sync()
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for table, stream in zip(tables, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            mi.mimose_op_muon_step(table, **HYPER, stream=torch.cuda.current_stream().cuda_stream)
        graphs.append(graph)
    again = [mi.MuonTable(es) for es in eager]
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        mi.mimose_op_muon_step(tables[2], **HYPER, stream=torch.cuda.current_stream().cuda_stream)
        sync()
        for table in again:
            mi.mimose_op_muon_step(table, **HYPER)
        sync()
        for ms, es in zip(sets, eager):
            for t, e in zip(ms, es):
                assert all(torch.equal(t[k], e[k]) for k in t)


def test_a_real_size():
    """A projection and a feed-forward block's matrix of the base model, against the definition on the GPU in 64 bits."""
    for shape in ((768, 768), (768, 3072), (3072, 768)):
        t = matrix(shape, shape[0])
        b = {k: x.double() for k, x in t.items()}
        mi.mimose_op_muon_step(mi.MuonTable([t]), **HYPER)
        m = HYPER["momentum"] * b["momentum"] + b["grad"]
        u = b["grad"] + HYPER["momentum"] * m
        x = u / (u.norm() + HYPER["eps"])
        for _ in range(5):
            A = x @ x.T if shape[0] <= shape[1] else x.T @ x
            B = om.COEFFICIENTS[1] * A + om.COEFFICIENTS[2] * A @ A
            x = om.COEFFICIENTS[0] * x + (B @ x if shape[0] <= shape[1] else x @ B)
        step = HYPER["rms"] * max(shape) ** 0.5 * x
        want = b["master"] - HYPER["lr"] * (step + HYPER["weight_decay"] * b["master"])
        sync()
        x64, off = om.orthogonalise(u.cpu().numpy(), HYPER["eps"], 5)
        assert np.allclose(x64, x.cpu().numpy(), atol=1e-9)
        assert float((t["master"].double() - want).norm()) <= HYPER["lr"] * HYPER["rms"] * max(shape) ** 0.5 * 3 * off
