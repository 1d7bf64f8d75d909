"""What the token losses and the update over a caller's tensors refuse, and that they say why.  Nothing is launched: a
call that is refused reads none of its pointers, so the addresses here are made up."""
import ctypes as C

import pytest

import paper_2209_02478_amd as mi

AT = 1 << 20            # an aligned address that nothing reads
LOGITS, GRAD, SMALL = AT, 1 << 40, 1 << 44


def refused(call, *args, **kw):
    with pytest.raises(mi.MimoseError) as e:
        call(*args, **kw)
    assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG
    return str(e.value)


def preference(**kw):
    a = dict(dtype=1, logits=LOGITS, ld=64, labels=SMALL, ends=None, pairs=2, L=3, ref_logp=SMALL, beta=0.1, smoothing=0.0, dlogits=GRAD,
             logp=SMALL, seq_logp=SMALL, margin=SMALL, loss=SMALL, T=12, V=60, workspace=AT, workspace_bytes=1 << 16)
    a.update(kw)
    return refused(mi.mimose_op_preference_loss, **a)


def policy(**kw):
    a = dict(dtype=1, logits=LOGITS, ld=64, labels=SMALL, old_logp=SMALL, ref_logp=SMALL, advantage=SMALL, weight=None, scale=1.0,
             clip_low=0.2, clip_high=0.2, kl_weight=0.1, dlogits=GRAD, rows=SMALL, stats=SMALL, T=12, V=60)
    a.update(kw)
    return refused(mi.mimose_op_policy_loss, **a)


def logprob(**kw):
    a = dict(dtype=1, logits=LOGITS, ld=64, labels=SMALL, logp=SMALL, T=12, V=60)
    a.update(kw)
    return refused(mi.mimose_op_token_logprob, **a)


@pytest.mark.parametrize("call", [preference, policy, logprob])
@pytest.mark.parametrize("wrong,why", [(dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype"), (dict(T=-1), "T >= 0"), (dict(V=0), "V >= 1"),
                                       (dict(ld=59), "ld >= V"), (dict(logits=None), "logits"), (dict(labels=None), "labels"),
                                       (dict(logits=LOGITS + 1), "aligned"), (dict(labels=SMALL + 2), "aligned"), (dict(ld=1 << 60), "ld too large")])
def test_rows_of_logits(call, wrong, why):
    assert why in call(**wrong)


@pytest.mark.parametrize("call", [preference, policy])
def test_gradients_that_overlap_the_logits(call):
    for at in (LOGITS + 2, LOGITS + 12 * 64 * 2 - 2, LOGITS - 12 * 64 * 2 + 2):
        assert "overlaps" in call(dlogits=at)
    assert "aligned" in call(dlogits=GRAD + 1)
    assert "aligned" in call(dtype=0, dlogits=GRAD + 2)


def test_preference():
    assert "pairs" in preference(pairs=0)
    assert "pairs" in preference(pairs=(1 << 24) + 1, ends=SMALL)
    assert "2 * pairs * L" in preference(T=11)
    assert "2 * pairs * L" in preference(L=-3)
    for name in ("ref_logp", "logp", "seq_logp", "margin", "loss"):
        assert "must be given" in preference(**{name: None})
    for beta in (float("nan"), float("inf")):
        assert "beta" in preference(beta=beta)
    for s in (-0.1, 1.1, float("nan")):
        assert "smoothing" in preference(smoothing=s)
    assert "workspace" in preference(workspace=None)
    assert "workspace" in preference(workspace=AT + 8)
    assert "workspace" in preference(workspace_bytes=mi.mimose_op_token_loss_workspace_bytes(12) - 1)


def test_policy():
    for name in ("old_logp", "advantage", "rows", "stats"):
        assert "must be given" in policy(**{name: None})
    assert "16-byte" in policy(rows=SMALL + 4)
    assert "scale" in policy(scale=float("inf"))
    for kw in (dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_low=float("nan")), dict(clip_high=-0.1), dict(clip_high=float("nan"))):
        assert "clip" in policy(**kw)
    for kl in (-0.1, float("nan"), float("inf")):
        assert "kl_weight" in policy(kl_weight=kl)
    assert "ref_logp" in policy(ref_logp=None)
    assert "workspace" in policy(workspace=AT, workspace_bytes=0)
    assert "workspace" in policy(workspace=AT + 4, workspace_bytes=1 << 16)


def test_logprob():
    assert "logp" in logprob(logp=None)
    assert "workspace" in logprob(workspace=AT, workspace_bytes=0)
    mi.mimose_op_token_logprob(1, None, 64, None, None, 0, 60)          # no rows: nothing to do


def tensor(**kw):
    t = mi.mimose_adamw_tensor(AT, 0, AT, AT, AT, AT, AT, 300, 1, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_table(bits):
    def bytes_of(*ts, state_bits=bits):
        return mi.mimose_op_adamw_table_bytes((mi.mimose_adamw_tensor * len(ts))(*ts), state_bits)

    assert bytes_of(tensor()) > 0 and bytes_of(tensor(), tensor(n=0, master=None)) >= bytes_of(tensor())
    assert "state_bits" in refused(bytes_of, tensor(), state_bits=16)
    assert "at least one" in refused(bytes_of)
    assert "negative" in refused(bytes_of, tensor(n=-1))
    for name in ("master", "grad", "m", "v"):
        assert "must be given" in refused(bytes_of, tensor(), tensor(**{name: None}))
    for name in ("master", "lowp", "grad", "m", "v"):
        assert "16-byte" in refused(bytes_of, tensor(**{name: AT + 4}))
    assert "too many" in refused(bytes_of, tensor(n=1 << 35))
    if bits == 8:
        for name in ("m_scale", "v_scale"):
            assert "m_scale and v_scale" in refused(bytes_of, tensor(**{name: None}))
            assert "m_scale and v_scale" in refused(bytes_of, tensor(**{name: AT + 2}))
    ts = (mi.mimose_adamw_tensor * 1)(tensor())
    need = mi.mimose_op_adamw_table_bytes(ts, bits)
    for device, n in ((None, need), (AT + 8, need), (AT, need - 1)):
        assert "16-byte aligned device memory" in refused(mi.mimose_op_adamw_table, ts, bits, device, n)


def test_adamw_step():
    good = mi.mimose_adamw_table(AT, 1, 1, 8, 0)
    assert "numbered from 1" in refused(mi.mimose_op_adamw_step, good, 0)
    for kw in (dict(lr=-1.0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(weight_decay=float("nan")), dict(lr=float("nan"))):
        assert "out of range" in refused(mi.mimose_op_adamw_step, good, 1, **kw)
    for bad in (mi.mimose_adamw_table(None, 1, 1, 8, 0), mi.mimose_adamw_table(AT, 0, 1, 8, 0), mi.mimose_adamw_table(AT, 1, -1, 8, 0),
                mi.mimose_adamw_table(AT, 1, 1, 4, 0)):
        assert "a table of" in refused(mi.mimose_op_adamw_step, bad, 1)
    lib = mi.load_library()
    assert lib.mimose_op_adamw_step(None, C.byref(mi.mimose_adamw_cfg(1e-3, 0.9, 0.99, 1e-8, 0.0)), 1, None) == mi.MIMOSE_ERR_INVALID_ARG
    assert lib.mimose_op_adamw_step(C.byref(good), None, 1, None) == mi.MIMOSE_ERR_INVALID_ARG
