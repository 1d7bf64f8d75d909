"""The smallest batches and the narrowest rows of the fine-tuning iterations, whose own numbers lie in memory that the step has anyway:
values against the oracle, a budget of the dry step's peak, and iterations of another loss right before and after.  Tolerances as in
test_gpu_finetune."""
import numpy as np
import pytest

import synthdata
import paper_2209_02478_amd as mi
from oracle import token_loss as tl
from test_gpu_finetune import oracle, oracle_logp, tols
from test_gpu_step import check_grads

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pre_ln", [0, 1])
@pytest.mark.parametrize("B,L,lengths", [(2, 1, None), (4, 1, None), (2, 2, [1, 2]), (18, 1, None), (6, 40, [40, 1, 1, 2, 1, 30])])
def test_against_the_oracle_in_the_dry_peak(dtype, pre_ln, B, L, lengths):
    shape = synthdata.ModelShape(2, 32, 1, 64, 100, 64, dtype, causal=pre_ln, pre_ln=pre_ln, gelu_tanh=pre_ln, head=1 - pre_ln)
    d = synthdata.shape_dict(shape)
    probe = mi.Mimose(d, 0, arena_bytes=64 << 20)
    probe.force_plan(0)
    peak, _ = probe.dry_step(B, L)
    probe.close()
    params = synthdata.make_params(shape, 3, perturb=True)
    m = mi.Mimose(d, peak)
    m.load_params(params)
    m.force_plan(0)
    tokens, labels = synthdata.make_batch(shape, B, L, 4)
    # labels that differ: with one label for both answers its column of the logits' gradient cancels in every sum over the rows, and
    # what is left is smaller than the roundings of what cancels
    labels = np.where(labels < 0, (11 * np.arange(B)[:, None] + 7) % 100, labels)
    n = None if lengths is None else np.array(lengths, np.int32)
    if lengths:
        for b in range(B):
            labels[b, lengths[b]:] = -1
    rng = np.random.default_rng(B + L)
    logp = oracle_logp(shape, params, tokens, labels, n)
    atol, gtol = tols(shape)
    ref = (logp.sum(1) + rng.standard_normal(B) * 3).astype(np.float32)
    old = (logp - rng.choice([-0.5, -0.1, 0.1, 0.5], size=(B, L))).astype(np.float32)
    kl_ref = (logp + rng.choice([-0.6, 0.6], size=(B, L))).astype(np.float32)
    adv, weight = rng.choice([-1.5, 0.7, 1.2], size=(B, L)).astype(np.float32), (rng.random((B, L)) / 8).astype(np.float32)
    kept = {}

    def pair(logits, lab):
        kept["pair"] = tl.preference_loss(logits, lab, [(b + 1) * L for b in range(B)], ref, 0.3, 0.1)
        return kept["pair"]["loss"], kept["pair"]["dlogits"]

    def policy(logits, lab):
        kept["policy"] = tl.policy_loss(logits, lab, old.ravel(), kl_ref.ravel(), adv.ravel(), weight.ravel(), 1.0, 0.2, 0.28, 0.1)
        return kept["policy"]["stats"][0], kept["policy"]["dlogits"]

    want_pair, grads_pair = oracle(shape, params, tokens, labels, n, pair)
    want_policy, grads_policy = oracle(shape, params, tokens, labels, n, policy)
    for _ in range(2):
        m.train_step(tokens, labels, n, wait=False)
        loss, margin, used, _ = m.train_step_preference(tokens, labels, ref, beta=0.3, smoothing=0.1, lengths=n)
        z_tol = 0.3 * 2 * np.sqrt(L) * atol
        assert used == peak and abs(loss - want_pair) <= z_tol and np.abs(margin - kept["pair"]["margin"]).max() <= z_tol
        check_grads(m.grads(), grads_pair, gtol)
        m.train_step_preference(tokens, labels, ref, lengths=n, wait=False)
        loss, stats, used, _ = m.train_step_policy(tokens, labels, old, adv, ref_logp=kl_ref, weight=weight, clip_low=0.2, clip_high=0.28,
                                                   kl_weight=0.1, lengths=n)
        total = float(np.abs(kept["policy"]["rows"][:, 1:]).sum())
        assert used == peak and loss == stats[0] and np.abs(stats - kept["policy"]["stats"]).max() <= 4 * atol * total
        check_grads(m.grads(), grads_policy, gtol)
        got = m.score(tokens, labels, n)
        assert np.abs(got - logp).max() <= atol
    m.close()
