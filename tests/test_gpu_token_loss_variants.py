"""Every variant of the row kernels, on rows that begin and end on a 16-byte address and on rows that do not, and both ways
a preference loss reads its rows; tolerances as in test_gpu_token_loss."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, TDT, host, quant, sync
from oracle import token_loss as tl
from test_gpu_token_loss import (check_gradient, check_logp, f32, i32, inputs, logits_of, lse_tol, policy_inputs, run_policy, run_preference,
                                 U)

pytestmark = pytest.mark.gpu

# columns in 16-byte chunks at the ends of each variant's range, and one chunk into the next
CHUNKS = [64, 65, 128, 129, 256, 257, 576, 577, 1152, 1153, 2304, 2305, 4608, 4609, 6656, 6657, 7168, 7169, 9216, 9217, 13312, 13313, 16384, 16385]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("chunks", CHUNKS)
def test_variant(dtype, chunks):
    n = 8 if dtype else 4
    T = 5
    # whole chunks; a tail of one column; rows on every address; the gradient on other addresses than the logits
    for V, ld, offset, grad_offset in ((chunks * n, chunks * n, 0, 0), (chunks * n - n + 1, chunks * n + n, 0, 0),
                                       ((chunks - 1) * n, (chunks - 1) * n + 1, 1, 1), ((chunks - 1) * n - 1, (chunks - 1) * n + 3, 0, 1)):
        x, labels, old, ref, adv, weight = policy_inputs(chunks + V, T, V, dtype)
        labels[0], labels[4] = 0, V - 1            # in the first and the last chunk
        x[0, 0] = x[4, V - 1] = 4.0                # (a label that is not far below its row's maximum)
        logp = tl.token_logprob(x, labels)[0]
        old = np.where(np.isfinite(old), logp - 0.1, old).astype(np.float32)
        ref = (logp + 0.3).astype(np.float32)
        bad = np.flatnonzero(~tl.scored_rows(labels, V))
        lg = logits_of(dtype, x, ld, offset, unscored=bad)
        buf = torch.full((T * ld + 16,), 9.0, dtype=TDT[dtype], device=DEV)
        d = buf[grad_offset:grad_offset + T * ld].view(T, ld)
        got = torch.full((T,), 3.0, device=DEV)
        mi.mimose_op_token_logprob(dtype, lg, ld, i32(labels), got, T, V)
        sync()
        check_logp(host(got), logp, V)
        args = (old, ref, adv, weight, 0.125, 0.2, 0.28, 0.05)
        want = tl.policy_loss(x, labels, *args)
        rows, _ = run_policy(dtype, lg, ld, labels, *args, d, T, V, None)
        slack = lse_tol(V) + 4 * U * np.abs(want["rows"][:, 0]) + 16 * U
        check_gradient(host(d), want, labels, V, dtype, 2 * slack)
        assert (buf[:grad_offset] == 9).all() and (buf[grad_offset + T * ld:] == 9).all()
        seq_ref = np.array([0.5, -0.5], np.float32)
        full = tl.preference_loss(x, labels, [2, 5], seq_ref, 0.05, 0.0)
        run_preference(dtype, lg, ld, labels, [2, 5], 1, 0, seq_ref, 0.05, 0.0, d, T, V)
        z_tol = 0.1 * (T * lse_tol(V) + 8 * U * np.abs(full["logp"]).sum()) + U * np.abs(full["margin"]).max()
        check_gradient(host(d), full, labels, V, dtype, z_tol + 16 * U)
        assert (buf[:grad_offset] == 9).all() and (buf[grad_offset + T * ld:] == 9).all()


@pytest.mark.parametrize("rows", [6670, 6671])
@pytest.mark.parametrize("ld", [50304, 50303])
def test_preference_rows_through_the_cache_and_past_it(rows, ld):
    """640 MB of logits are read through the caches, more are not (50304 columns in bf16: 6670 rows and 6671).  A few rows of either
    sequence are scored, the first and the last among them."""
    V = 50257
    assert (6670 * 50304 * 2 <= 640 << 20) and (6671 * 50304 * 2 > 640 << 20)
    lg = torch.full((rows * ld,), 1.0, dtype=torch.bfloat16, device=DEV).view(rows, ld)
    at = [0, 1, 3000, 3334, 3335, 5000, rows - 2, rows - 1]
    rng, x, labels = inputs(rows, len(at), V, 1)
    labels[:] = rng.integers(0, V, len(at))
    lg[at, :V] = torch.tensor(x.astype(np.float32)).to(torch.bfloat16).to(DEV)
    all_labels = np.full(rows, -1, np.int32)
    all_labels[at] = labels
    ref = np.array([-30.0, -31.0], np.float32)
    want = tl.preference_loss(x, labels, [4, 8], ref, 0.1, 0.1)
    d = torch.full_like(lg, 5.0)
    out = run_preference(1, lg, ld, all_labels, [3335, rows], 1, 0, ref, 0.1, 0.1, d, rows, V)
    check_logp(host(out["logp"])[at], want["logp"], V)
    seq_tol = 8 * lse_tol(V) + 8 * U * np.abs(want["logp"]).sum()
    z_tol = 0.2 * seq_tol + U * np.abs(want["margin"]).max()
    assert np.abs(host(out["margin"]) - want["margin"]).max() <= z_tol
    assert abs(float(out["loss"]) - want["loss"]) <= z_tol + 8 * U * want["loss"]
    check_gradient(host(d[at]), want, labels, V, 1, z_tol + 16 * U)
    d[at] = 0
    assert not d.any()


def test_infinities_and_nan_stay_in_their_rows():
    """A NaN, or +inf, among a scored row's logits makes that row NaN and, in the preference loss, its pair; nothing else."""
    for V, ld in ((500, 512), (20000, 20000), (140000, 140032)):
        T = 8
        x = quant(np.random.default_rng(V).standard_normal((T, V)), 1)
        lg = logits_of(1, x, ld)
        lg[2, V // 2], lg[5, V - 1] = float("nan"), float("inf")
        labels = np.arange(T, dtype=np.int32)
        logp = torch.empty(T, device=DEV)
        mi.mimose_op_token_logprob(1, lg, ld, i32(labels), logp, T, V)
        sync()
        assert np.array_equal(np.isnan(host(logp)), np.isin(np.arange(T), (2, 5)))
        d = torch.empty_like(lg)
        zeros = np.zeros(T, np.float32)
        run_policy(1, lg, ld, labels, host(logp).astype(np.float32), None, zeros + 1, None, 1.0, 0.2, 0.2, 0.0, d, T, V, None)
        assert np.array_equal(np.isnan(host(d)[:, :V]).any(1), np.isin(np.arange(T), (2, 5))) and not d[:, V:].any()
        lg[5, V - 1] = 0.0
        run_preference(1, lg, ld, labels, None, 2, 2, zeros[:4], 0.1, 0.0, d, T, V)
        assert np.array_equal(np.isnan(host(d)[:, :V]).any(1), np.arange(T) < 4) and not d[:, V:].any()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("lengths", [[3, 0], [0, 0, 1, 5], [200, 1, 0, 300] * 4, [1] * 18, [400, 700], [70] * 16 + [2, 3], [64, 65] * 8])
@pytest.mark.parametrize("grad", [False, True])
def test_preference_sums(dtype, lengths, grad):
    """Up to eight pairs and more, few rows and many, sequences without rows, rows behind the last end: the pairs' numbers come out of
    the gradient's launch, or out of one of their own, and are the oracle's either way."""
    P, V, ld = len(lengths) // 2, 700, 704
    ends = np.cumsum(lengths)
    T = int(ends[-1]) + 3
    rng, x, labels = inputs(T, T, V, dtype)
    if sum(lengths) == 0:
        labels[:] = -1
    logp = tl.token_logprob(x, labels)[0]
    sums = np.array([logp[a:b].sum() for a, b in zip(np.concatenate([[0], ends[:-1]]), ends)])
    ref = (sums + rng.standard_normal(2 * P)).astype(np.float32)
    want = tl.preference_loss(x, labels, ends, ref, 0.2, 0.1)
    lg = logits_of(dtype, x, ld)
    d = torch.full_like(lg, 9.0) if grad else None
    out = run_preference(dtype, lg, ld, labels, ends, P, 0, ref, 0.2, 0.1, d, T, V)
    check_logp(host(out["logp"]), want["logp"], V)
    seq_tol = max(lengths) * lse_tol(V) + 8 * U * np.abs(want["logp"]).sum()
    assert np.abs(host(out["seq"]) - want["seq_logp"]).max() <= seq_tol
    z_tol = 0.4 * seq_tol + U * np.abs(want["margin"]).max()
    assert np.abs(host(out["margin"]) - want["margin"]).max() <= z_tol
    assert abs(float(out["loss"]) - want["loss"]) <= z_tol + 8 * U * want["loss"]
    if grad:
        check_gradient(host(d), want, labels, V, dtype, z_tol + 16 * U)
