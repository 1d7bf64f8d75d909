"""What the update with orthogonalised steps refuses, and how it lays a list out: host code alone, no address is read."""
import ctypes as C

import pytest

import paper_2209_02478_amd as mi

AT = [1 << k for k in range(30, 46)]


def entry(i=0, rows=10, cols=20, **kw):
    a = dict(master=AT[4 * i], lowp=AT[4 * i + 1], grad=AT[4 * i + 2], momentum=AT[4 * i + 3], rows=rows, cols=cols)
    a.update(kw)
    return a


def array(*entries):
    m = (mi.mimose_muon_matrix * len(entries))()
    for e, x in zip(m, entries):
        for k, v in x.items():
            setattr(e, k, v)
    return m


def refused(call, *args, **kw):
    with pytest.raises(mi.MimoseError) as e:
        call(*args, **kw)
    assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG
    return str(e.value)


@pytest.mark.parametrize("wrong,why", [
    (dict(rows=-1), "side"), (dict(cols=(1 << 20) + 1), "side"), (dict(master=None), "given"), (dict(grad=None), "given"),
    (dict(momentum=None), "given"), (dict(master=AT[0] + 4), "16-byte"), (dict(grad=AT[2] + 8), "16-byte"), (dict(momentum=AT[3] + 4), "16-byte"),
    (dict(lowp=AT[1] + 2), "16-byte"), (dict(momentum=AT[0]), "belongs"), (dict(grad=AT[0] + 16), "belongs"), (dict(lowp=AT[3] + 784), "belongs"),
    (dict(rows=1 << 20, cols=1 << 20), "too many"), (dict(rows=1 << 19, cols=1 << 19, master=1 << 50, grad=1 << 51, momentum=1 << 52, lowp=0), "too many")])
def test_lists(wrong, why):
    assert why in refused(mi.mimose_op_muon_table_bytes, array(entry(**wrong)), 1)
    assert why in refused(mi.mimose_op_muon_table, array(entry(**wrong)), 1, AT[12], 1 << 20)


def test_lists_of_two():
    assert mi.mimose_op_muon_table_bytes(array(entry(0), entry(1)), 1) > 0
    assert "belongs" in refused(mi.mimose_op_muon_table_bytes, array(entry(0), entry(0)), 1)
    assert "belongs" in refused(mi.mimose_op_muon_table_bytes, array(entry(0), entry(1, master=AT[0] + 10 * 20 * 4 - 16)), 1)
    assert mi.mimose_op_muon_table_bytes(array(entry(0), entry(1, master=AT[0] + 10 * 20 * 4)), 1) > 0
    assert mi.mimose_op_muon_table_bytes(array(entry(0), entry(1, grad=AT[2])), 1) > 0          # one gradient may serve two
    assert mi.mimose_op_muon_table_bytes(array(entry(0, rows=0, master=None)), 1) > 0           # nothing in it: nothing looked at
    for parts in (0, 65, -1):
        assert "parts" in refused(mi.mimose_op_muon_table_bytes, array(entry()), parts)
    assert "at least one" in refused(mi.mimose_op_muon_table_bytes, (mi.mimose_muon_matrix * 0)(), 1)


def test_table():
    m = array(entry())
    need = mi.mimose_op_muon_table_bytes(m, 1)
    for device, n in ((None, need), (AT[12] + 8, need), (AT[12], need - 1)):
        assert "mimose_op_muon_table_bytes" in refused(mi.mimose_op_muon_table, m, 1, device, n)


def table(**kw):
    t = mi.mimose_muon_table()
    t.device, t.workspace_bytes, t.matrices, t.parts = AT[0], 1 << 16, 1, 1
    t.units[0][0] = t.units[1][0] = 1
    for k, v in kw.items():
        setattr(t, k, v)
    return t


@pytest.mark.parametrize("wrong,why", [
    (dict(lr=-1.0), "hyper"), (dict(lr=float("nan")), "hyper"), (dict(lr=float("inf")), "hyper"), (dict(momentum=1.0), "hyper"), (dict(momentum=-0.1), "hyper"),
    (dict(weight_decay=-1.0), "hyper"), (dict(rms=-0.1), "hyper"), (dict(eps=0.0), "hyper"), (dict(eps=float("inf")), "hyper"),
    (dict(iterations=0), "iterations"), (dict(iterations=65), "iterations"), (dict(workspace=None), "workspace"),
    (dict(workspace=AT[1] + 8), "workspace"), (dict(workspace_bytes=(1 << 16) - 1), "workspace")])
def test_steps(wrong, why):
    assert why in refused(mi.mimose_op_muon_step, table(), **(dict(workspace=AT[1], workspace_bytes=1 << 16) | wrong))


def test_tables_that_are_none():
    for kw in (dict(device=None), dict(matrices=-1), dict(parts=0), dict(parts=65)):
        assert "table" in refused(mi.mimose_op_muon_step, table(**kw), workspace=AT[1], workspace_bytes=1 << 16)
    t = table(parts=2)
    t.units[0][1] = 0
    assert "table" in refused(mi.mimose_op_muon_step, t, workspace=AT[1], workspace_bytes=1 << 16)
