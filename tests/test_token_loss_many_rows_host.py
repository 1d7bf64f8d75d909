"""Calls with more rows than one launch takes, up to the last row count that the entry points know: the launches end, and there are
as many as the rows need (on the stand-in for the HIP runtime of test_launch_errors, which launches nothing)."""
import pytest

from test_launch_choice import run
from test_launch_errors import runtime  # noqa: F401
from test_token_loss_launches import SETUP


@pytest.mark.parametrize("T", [1 << 20, (1 << 20) + 1, (1 << 31) - (1 << 20), (1 << 31) - (1 << 20) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("V", [1, 140000])              # held rows and long ones
def test_launches(runtime, T, V):  # noqa: F811
    run(runtime, SETUP + """
    T, V = map(int, sys.argv[2:])
    want = -(-T // (1 << 20))
    names = launched(lambda: mi.mimose_op_token_logprob(1, at, V, at, at, T, V))
    assert len(names) == want and all("token_rows" in n for n in names), (len(names), want)
    names = policy(1, V, V, at, 1 << 60, T)
    assert len(names) == want + 1 and "policy_stats" in names[-1], (len(names), want)
    names = preference(1, V, V, T, None)
    assert len(names) == want + 1 and "few_pairs" in names[-1], (len(names), want)
    names = preference(1, V, V, T, 1 << 60)
    grads = [n for n in names if "pair_grad" in n]
    parts = -(-V // (2048 if "Lb1E" in grads[0].split("pair_grad_kernel")[1][:8] else 4096))
    assert len(names) == want + 1 + len(grads) and len(grads) == -(-T // ((1 << 23) // parts)), (len(names), want, parts)
    """, T, V)
