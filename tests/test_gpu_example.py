"""examples/finetune.py on the smallest configuration: it runs, keeps to its budget, and learns its batches."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", ["8", "32"])
def test_finetune(bits):
    import finetune
    r = finetune.main(["--model", "tiny", "--pairs", "2", "--steps", "30", "--state-bits", bits, "--lr", "1e-3", "--budget-frac", "0.9"])
    assert r["peak"] <= r["budget"]
    for first, last in r["preference"].values():       # ten updates a batch, each of which can be told apart by its tokens
        assert abs(first - np.log(2)) < 0.2 and last < 0.5 * first
    assert all(np.isfinite(x).all() for x in r["policy"])
    losses = [x[0] for x in r["policy"]]
    assert np.mean(losses[1::2]) < np.mean(losses[0::2])           # the second update from one scoring starts lower
