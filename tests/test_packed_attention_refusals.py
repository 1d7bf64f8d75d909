"""What packed attention refuses, and that it says why.  Nothing is launched: the addresses are made up."""
import pytest

import paper_2209_02478_amd as mi

AT = [1 << k for k in range(30, 44)]     # addresses far from each other that nothing reads


def fwd(**kw):
    a = dict(dtype=1, q=AT[0], ldq=256, k=AT[1], ldk=128, v=AT[2], ldv=128, out=AT[3], ldo=256, lse=AT[4], ends=AT[5], n_seq=2, T=10,
             n_heads=4, n_kv_heads=2, head_dim=64, causal=1, scale=0.125)
    a.update(kw)
    return refused(mi.mimose_op_packed_attention_fwd, a)


def bwd(**kw):
    a = dict(dtype=1, q=AT[0], ldq=256, k=AT[1], ldk=128, v=AT[2], ldv=128, out=AT[3], ldo=256, lse=AT[4], dout=AT[6], lddo=256,
             dq=AT[7], lddq=256, dk=AT[8], lddk=128, dv=AT[9], lddv=128, ends=AT[5], n_seq=2, T=10, n_heads=4, n_kv_heads=2, head_dim=64,
             causal=1, scale=0.125, workspace=AT[10], workspace_bytes=1 << 20)
    a.update(kw)
    return refused(mi.mimose_op_packed_attention_bwd, a)


def refused(call, a):
    with pytest.raises(mi.MimoseError) as e:
        call(**a)
    assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG
    return str(e.value)


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("wrong,why", [
    (dict(dtype=2), "dtype"), (dict(T=-1), "T >= 0"), (dict(n_seq=-1), "n_seq"), (dict(n_heads=5), "multiple"), (dict(n_heads=0), "multiple"),
    (dict(n_kv_heads=0), "multiple"), (dict(head_dim=48), "head_dim"), (dict(head_dim=256), "head_dim"), (dict(scale=0.0), "scale"),
    (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"), (dict(ends=None), "ends"),
    (dict(ends=AT[5] + 2), "ends"), (dict(q=None), "given"), (dict(k=None), "given"), (dict(v=None), "given"), (dict(out=None), "given"),
    (dict(lse=None), "given"), (dict(lse=AT[4] + 2), "lse"), (dict(ldq=255), "leading"), (dict(ldk=120), "leading"), (dict(ldv=1 << 21), "leading"),
    (dict(ldo=250), "leading"), (dict(ldq=260), "16-byte"), (dict(q=AT[0] + 8), "16-byte"), (dict(v=AT[2] + 2), "16-byte"),
    (dict(T=(1 << 31) - 1), "too many"), (dict(n_seq=1 << 30), "too many")])
def test_arguments(call, wrong, why):
    assert why in call(**wrong)


def test_of_fp32():
    assert "16-byte" in fwd(dtype=0, ldq=258)
    assert "leading" in fwd(dtype=0, ldk=124)


def test_what_is_written_overlaps():
    for at in (AT[0], AT[0] + 16, AT[1], AT[2] + 128 * 2 * 9, AT[5] - 16):
        assert "overlaps" in fwd(out=at)
    for at in (AT[3], AT[0] + 256, AT[5]):
        assert "overlaps" in fwd(lse=at)
    # rows of one pitch beside each other: columns that meet, and that begin in one row and end in the next
    assert "overlaps" in fwd(q=AT[0], ldq=512, out=AT[0] + 256 * 2 - 16, ldo=512)
    assert "overlaps" in fwd(q=AT[0] + 512, ldq=512, out=AT[0] + 16, ldo=512)
    assert "overlaps" in bwd(dq=AT[0])
    assert "overlaps" in bwd(dk=AT[1], lddk=128)
    assert "overlaps" in bwd(dv=AT[8])
    assert "overlaps" in bwd(workspace=AT[7])
    assert "overlaps" in bwd(dq=AT[4])


def test_scratch():
    need = mi.mimose_op_packed_attention_bwd_workspace_bytes(10, 4, 2, 64)
    assert need >= 10 * 4 * 4
    for wrong in (dict(workspace=None), dict(workspace=AT[10] + 8), dict(workspace_bytes=need - 1)):
        assert "workspace" in bwd(**wrong)


def test_nothing_to_do():
    """No rows or no sequences: nothing is launched and no operand looked at."""
    for kw in (dict(T=0), dict(n_seq=0)):
        a = dict(dtype=1, q=None, ldq=0, k=None, ldk=0, v=None, ldv=0, out=None, ldo=0, lse=None, ends=AT[5], n_seq=2, T=10, n_heads=4,
                 n_kv_heads=2, head_dim=64, causal=1, scale=0.125)
        a.update(kw)
        mi.mimose_op_packed_attention_fwd(**a)
