"""Rows of a policy loss that their weight leaves out, with logits that are not finite: such a row gives the loss nothing and its
gradient is zeros, whatever it holds, and every other row has the bits that it has beside a finite one."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, TDT
from test_gpu_token_loss import logits_of, policy_inputs, run_policy

pytestmark = pytest.mark.gpu

# a wave for a row, several waves, rows off 16 bytes, rows too long to be held
SHAPES = [(1, 1, 0), (7, 7, 1), (1000, 1024, 0), (5000, 5056, 1), (50257, 50304, 0), (150001, 150016, 0)]
FILLS = {"nan": [np.nan], "inf": [np.inf, 0.0], "-inf": [-np.inf], "mixed": [np.nan, np.inf, -np.inf, 3.0]}


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V,ld,offset", SHAPES)
@pytest.mark.parametrize("fill", list(FILLS))
def test_rows_of_weight_zero(dtype, V, ld, offset, fill):
    T, out = 9, [0, 3, 8]
    x, labels, old, ref, adv, weight = policy_inputs(V, T, V, dtype)
    labels[:] = np.arange(T) % V
    weight[out], old[out], adv[out] = 0.0, 1.0, 1.0
    weight[[1, 2, 4, 5, 6, 7]] = 0.5
    args = (old, ref, adv, weight, 0.125, 0.2, 0.28, 0.05)
    finite = logits_of(dtype, x, ld, offset)
    bad = finite.clone() if offset == 0 else logits_of(dtype, x, ld, offset)
    values = torch.tensor(FILLS[fill]).repeat(-(-V // len(FILLS[fill])))[:V].to(TDT[dtype]).to(DEV)
    for t in out:
        bad[t, :V] = values
    d0, d1, d2 = (torch.full((T, ld), 9.0, dtype=TDT[dtype], device=DEV) for _ in range(3))
    rows0, stats0 = run_policy(dtype, finite, ld, labels, *args, d0, T, V, None)
    rows1, stats1 = run_policy(dtype, bad, ld, labels, *args, d1, T, V, None)
    shifted = torch.full((T * ld + 16,), 9.0, dtype=TDT[dtype], device=DEV)[3:3 + T * ld].view(T, ld)   # on other addresses than the logits
    run_policy(dtype, bad, ld, labels, *args, shifted, T, V, None)
    run_policy(dtype, bad, ld, labels, *args, bad, T, V, None)
    kept = [t for t in range(T) if t not in out]
    assert torch.equal(stats0, stats1) and torch.equal(rows0[:, 1:], rows1[:, 1:]) and torch.equal(rows0[kept], rows1[kept])
    assert not rows1[out, 1:].any()
    assert not d1[out].any() and torch.equal(d1, d0) and torch.equal(d1, bad) and torch.equal(d1, shifted)


def test_a_scale_of_zero():
    """Every row is left out."""
    V, ld, T = 1000, 1024, 5
    x, labels, old, ref, adv, weight = policy_inputs(1, T, V, 1)
    labels[:] = 3
    lg = logits_of(1, x, ld)
    lg[2] = float("nan")
    d = torch.full_like(lg, 9.0)
    rows, stats = run_policy(1, lg, ld, labels, old, ref, adv, weight, 0.0, 0.2, 0.28, 0.05, d, T, V, None)
    assert not d.any() and not stats.any() and not rows[:, 1:].any()
