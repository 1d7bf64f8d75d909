"""Iterations with a preference or a policy loss, scoring, and the update with moments in 8 bits, through the executor.

Gradients are compared as those of the cross-entropy step (tests/test_gpu_step.py) are: relative L2 error of each tensor
within 1e-3 (fp32).  In bf16 that is 2e-2 there; here the softmax parts of a pair's sequences, or of advantages of either
sign, cancel to a good part while their roundings do not, so the same roundings are up to sqrt(2) larger beside what is
left: 3e-2.  Log-probabilities in bf16: the logits of these models are below 1.5 in magnitude and rounded to bf16 (2^-8
relative), and what they are made of is off by about 1 %: 2e-2."""
import numpy as np
import pytest

import synthdata
import paper_2209_02478_amd as mi
from oracle import model as om
from oracle import optimizer8 as o8
from oracle import token_loss as tl
from test_gpu_step import SMALL, MiB, check_grads

pytestmark = pytest.mark.gpu

NAMES = ["fp32_preln_causal", "fp32_postln", "bf16_preln_causal", "bf16_postln"]
LENGTHS = [33, 20, 7, 33, 1, 30]


def model(name, **kw):
    shape = SMALL[name]
    params = synthdata.make_params(shape, 11, perturb=True)
    m = mi.Mimose(synthdata.shape_dict(shape), 0, arena_bytes=256 * MiB, **kw)
    m.load_params(params)
    m.force_plan(0)
    return shape, params, m


def batch(shape, padded):
    """Six samples; the first third of a sample is its prompt, not scored."""
    if padded:
        tokens, labels, lengths = synthdata.make_padded_batch(shape, LENGTHS, 12)
    else:
        (tokens, labels), lengths = synthdata.make_batch(shape, 6, 33, 12), None
    labels = labels.copy()
    for b in range(6):
        labels[b, :(LENGTHS[b] if padded else 33) // 3] = -1
    return tokens, labels, lengths


def oracle(shape, params, tokens, labels, lengths, loss_fn):
    cfg = om.Cfg.from_shape(synthdata.shape_dict(shape))
    if shape.dtype == "bf16":
        params = {k: om.round_to_bf16(v) for k, v in params.items()}
    return om.train_step(cfg, params, tokens, labels, lengths=lengths, loss_fn=loss_fn)


def oracle_logp(shape, params, tokens, labels, lengths):
    kept = {}

    def fn(logits, lab):
        kept["logp"] = tl.token_logprob(logits, lab)[0]
        return 0.0, np.zeros_like(logits)

    oracle(shape, params, tokens, labels, lengths, fn)
    return kept["logp"].reshape(tokens.shape)


def tols(shape):
    return (1e-4, 1e-3) if shape.dtype == "fp32" else (2e-2, 3e-2)


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_score(name, padded):
    shape, params, m = model(name)
    tokens, labels, lengths = batch(shape, padded)
    want = oracle_logp(shape, params, tokens, labels, lengths)
    loss0, peak0, _ = m.train_step(tokens, labels, lengths)
    grads0 = m.grads()
    m.set_dropout(0.3, 0.2, seed=5)                    # a model is scored without it
    before = m.stats()
    got = m.score(tokens, labels, lengths)
    assert m.stats() == before
    m.set_dropout(0.0)
    assert np.abs(got - want).max() <= tols(shape)[0]
    assert not got[labels < 0].any()
    assert np.array_equal(m.score(tokens, labels, lengths), got)
    loss1, peak1, _ = m.train_step(tokens, labels, lengths)
    assert (loss0, peak0) == (loss1, peak1)
    grads1 = m.grads()
    assert all(np.array_equal(grads0[k], grads1[k]) for k in grads0)
    # the mean cross-entropy is minus the mean of the log-probabilities
    n = (labels >= 0).sum()
    assert abs(loss0 + got.sum(dtype=np.float64) / n) <= 1e-5 * abs(loss0)
    m.close()


@pytest.mark.parametrize("smoothing", [0.0, 0.1])
@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_preference_step(name, padded, smoothing):
    shape, params, m = model(name)
    tokens, labels, lengths = batch(shape, padded)
    L = tokens.shape[1]
    logp = oracle_logp(shape, params, tokens, labels, lengths)
    ref = (logp.sum(1) + np.array([1.0, -2.0, 0.5, 0.0, -3.0, 2.0])).astype(np.float32)
    kept = {}

    def fn(logits, lab):
        kept.update(tl.preference_loss(logits, lab, [(b + 1) * L for b in range(6)], ref, 0.3, smoothing))
        return kept["loss"], kept["dlogits"]

    want, RG = oracle(shape, params, tokens, labels, lengths, fn)
    loss, margin, peak, plan = m.train_step_preference(tokens, labels, ref, beta=0.3, smoothing=smoothing, lengths=lengths)
    G = m.grads()
    atol, gtol = tols(shape)
    # a margin is beta times the errors of two sums of up to 33 log-probabilities, of random sign
    assert np.abs(margin - kept["margin"]).max() <= 0.3 * 2 * np.sqrt(33) * atol
    assert abs(loss - want) <= 0.3 * 2 * np.sqrt(33) * atol
    check_grads(G, RG, gtol)
    # any plan, queued or waited for: the same bits
    for p in range(1 << shape.n_layers):
        m.force_plan(p)
        again, margin2, _, got = m.train_step_preference(tokens, labels, ref, beta=0.3, smoothing=smoothing, lengths=lengths)
        assert got == p and again == loss and np.array_equal(margin, margin2)
        H = m.grads()
        assert all(np.array_equal(G[k], H[k]) for k in G), p
    m.train_step_preference(tokens, labels, ref, beta=0.3, smoothing=smoothing, lengths=lengths, wait=False)
    assert m.sync_loss() == loss
    H = m.grads()
    assert all(np.array_equal(G[k], H[k]) for k in G)
    m.close()


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("name", NAMES)
def test_policy_step(name, padded, weighted):
    shape, params, m = model(name)
    tokens, labels, lengths = batch(shape, padded)
    B, L = tokens.shape
    rng = np.random.default_rng(3)
    logp = oracle_logp(shape, params, tokens, labels, lengths)
    # ratios well off the bounds of 0.8 and 1.28 (logarithms -0.22 and 0.25), which an error of 2e-2 then does not cross
    old = (logp - rng.choice([-0.5, -0.1, 0.0, 0.1, 0.5], size=(B, L))).astype(np.float32)
    ref = (logp + rng.choice([-0.6, -0.3, 0.3, 0.6], size=(B, L))).astype(np.float32)
    adv = rng.choice([-1.5, -0.5, 0.7, 1.2], size=(B, L)).astype(np.float32)
    weight = (rng.random((B, L)) / 40).astype(np.float32) if weighted else None
    n = int((labels >= 0).sum())
    kl = 0.1 if weighted else 0.0
    kept = {}

    def fn(logits, lab):
        kept.update(tl.policy_loss(logits, lab, old.ravel(), ref.ravel() if weighted else None, adv.ravel(),
                                   None if weight is None else weight.ravel(), 1.0 if weighted else 1.0 / n, 0.2, 0.28, kl))
        return kept["stats"][0], kept["dlogits"]

    want, RG = oracle(shape, params, tokens, labels, lengths, fn)
    kw = dict(ref_logp=ref if weighted else None, weight=weight, clip_low=0.2, clip_high=0.28, kl_weight=kl, lengths=lengths)
    loss, stats, _, _ = m.train_step_policy(tokens, labels, old, adv, **kw)
    G = m.grads()
    atol, gtol = tols(shape)
    total = float(np.abs(kept["rows"][:, 1:]).sum())
    assert loss == stats[0] and np.abs(stats - kept["stats"]).max() <= 4 * atol * total
    check_grads(G, RG, gtol)
    m.force_plan(1)
    again, stats2, _, _ = m.train_step_policy(tokens, labels, old, adv, **kw)
    H = m.grads()
    assert again == loss and np.array_equal(stats, stats2) and all(np.array_equal(G[k], H[k]) for k in G)
    m.train_step_policy(tokens, labels, old, adv, wait=False, **kw)
    assert m.sync_loss() == loss
    m.close()


def test_objectives_in_turn_change_nothing_of_each_other():
    """Cross-entropy, preference, policy and scores queued behind one another, more steps than there are staging buffers."""
    shape, params, m = model("bf16_preln_causal")
    tokens, labels, lengths = batch(shape, True)
    rng = np.random.default_rng(1)
    ref = rng.standard_normal(6).astype(np.float32) * 20 - 100
    old, adv = (rng.standard_normal(tokens.shape).astype(np.float32) - 6 for _ in range(2))
    calls = [lambda w: m.train_step(tokens, labels, lengths, wait=w),
             lambda w: m.train_step_preference(tokens, labels, ref, lengths=lengths, wait=w),
             lambda w: m.train_step_policy(tokens, labels, old, adv, lengths=lengths, wait=w)]
    alone = []
    for call in calls:
        loss = call(True)[0]
        alone.append((loss, m.grads()))
    scores = m.score(tokens, labels, lengths)
    for k in (0, 1, 2, 2, 1, 0, 2, 0, 1):
        for j in (0, 1, 2):
            calls[(j + k) % 3](False)
        assert np.array_equal(m.score(tokens, labels, lengths), scores)
        last = (2 + k) % 3
        assert m.sync_loss() == alone[last][0]
        G = m.grads()
        assert all(np.array_equal(G[n], alone[last][1][n]) for n in G)
    m.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_update_with_moments_in_8_bits(dtype):
    """Parameters against the oracle's update of the library's own gradients, from the first update on, and the bytes that it saves."""
    hyper = dict(lr=2e-3, beta1=0.9, beta2=0.98, eps=1e-7, weight_decay=0.05)
    h32 = {k: float(np.float32(v)) for k, v in hyper.items()}
    shape = synthdata.ModelShape(2, 64, 2, 256, 1000, 64, dtype)
    params = synthdata.make_params(shape, 5, perturb=True)
    fixed = {}
    for bits in (32, 8):
        m = mi.Mimose(synthdata.shape_dict(shape), 0, arena_bytes=64 * MiB)
        m.load_params(params)
        m.optimizer_init(state_bits=bits, **hyper)
        fixed[bits] = m.stats()["fixed_bytes"]
        if bits == 32:
            m.close()
    n = sum(v.size for v in params.values())
    assert 6 * n - n / 32 - 1024 * len(params) <= fixed[32] - fixed[8] <= 6 * n
    bf16 = dtype == "bf16"
    state = {k: dict(p=(om.round_to_bf16(v) if bf16 else v).astype(np.float64).ravel(), m=np.zeros(v.size, np.uint8), v=np.zeros(v.size, np.uint8),
                     ms=np.zeros(-(-v.size // 256)), vs=np.zeros(-(-v.size // 256))) for k, v in params.items()}
    for step in range(1, 5):
        tokens, labels = synthdata.make_batch(shape, 3, 17 + 5 * step, 40 + step)
        m.train_step(tokens, labels)
        G = m.grads()
        m.optimizer_step()
        got = m.params()
        for k, s in state.items():
            wd = h32["weight_decay"] if params[k].ndim >= 2 else 0.0
            r = o8.step(s["p"], G[k].astype(np.float64).ravel(), s["m"], s["v"], s["ms"], s["vs"], step, **dict(h32, weight_decay=wd))
            s.update(p=r["p"], m=r["m"], v=r["v"], ms=r["m_scale"], vs=r["v_scale"])
            a, b = got[k].ravel(), (om.round_to_bf16(r["p"].astype(np.float32)) if bf16 else r["p"])
            # a code that falls to the other side of a rounding (one in ten thousand) moves later updates by up to an eighth
            # of one; all others follow the oracle to the rounding of the master and of bf16
            tol = 1e-6 * step * (np.abs(b) + hyper["lr"] * 10) + (2.0 ** -7 * np.abs(b) if bf16 else 0)
            off = np.abs(a - b) > tol
            assert off.mean() <= 2e-3, (k, step, off.mean())
            assert np.abs(a - b).max() <= hyper["lr"] * step + (2.0 ** -7 * np.abs(b).max() if bf16 else 0)
    m.close()


def test_refusals():
    shape, params, m = model("fp32_preln_causal")
    tokens, labels = synthdata.make_batch(shape, 4, 9, 1)
    odd = tokens[:3], labels[:3]
    z = np.zeros((4, 9), np.float32)

    def refused(call, *args, **kw):
        with pytest.raises(mi.MimoseError) as e:
            call(*args, **kw)
        assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG
        return str(e.value)

    assert "even" in refused(m.train_step_preference, *odd, np.zeros(3))
    assert "beta" in refused(m.train_step_preference, tokens, labels, np.zeros(4), beta=float("nan"))
    assert "smoothing" in refused(m.train_step_preference, tokens, labels, np.zeros(4), smoothing=2.0)
    assert "clip_low" in refused(m.train_step_policy, tokens, labels, z, z, clip_low=-1.0)
    assert "ref_logp" in refused(m.train_step_policy, tokens, labels, z, z, kl_weight=0.1)
    assert "label" in refused(m.score, tokens, np.full_like(labels, shape.vocab))
    assert "length" in refused(m.score, tokens, labels, np.array([0, 1, 2, 3]))
    assert "state_bits" in refused(m.optimizer_init, state_bits=16)
    with pytest.raises(ValueError):
        m.train_step_preference(tokens, labels, np.zeros(3))
    with pytest.raises(ValueError):
        m.train_step_policy(tokens, labels, z[:3], z)
    assert np.isfinite(m.train_step(tokens, labels)[0])            # the context stays usable
    m.close()


def test_a_budget_that_a_score_or_a_step_does_not_fit():
    shape = SMALL["bf16_preln_causal"]
    cal = mi.Mimose(synthdata.shape_dict(shape), 0, device=None)
    fixed = cal.stats()["fixed_bytes"]
    cal.close()
    m = mi.Mimose(synthdata.shape_dict(shape), fixed + (256 << 10))
    m.load_params(synthdata.make_params(shape, 1))
    tokens, labels = synthdata.make_batch(shape, 8, 64, 1)
    for call in (lambda: m.score(tokens, labels), lambda: m.train_step_preference(tokens, labels, np.zeros(8))):
        with pytest.raises(mi.MimoseError) as e:
            call()
        assert e.value.code == mi.MIMOSE_ERR_OOM_BUDGET
    small = tokens[:1, :4], labels[:1, :4]
    assert np.isfinite(m.score(*small)).all()
    m.close()
