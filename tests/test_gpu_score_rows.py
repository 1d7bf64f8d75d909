"""The log-probabilities of a score are those of the iteration that they are compared with, bit for bit: with the score as the old
policy and as the reference every ratio is exactly 1 and the KL term exactly 0."""
import numpy as np
import pytest

import synthdata
import paper_2209_02478_amd as mi
from test_gpu_step import SMALL, MiB

pytestmark = pytest.mark.gpu

LENGTHS = [33, 20, 7, 33, 1, 30, 2, 9]


SHAPES = {k: SMALL[k] for k in ("fp32_preln_causal", "fp32_postln", "bf16_preln_causal", "bf16_postln")}
# products of several tiles: their sums depend on how many rows there are
SHAPES["fp32_preln_causal_256"] = synthdata.ModelShape(2, 256, 4, 1024, 1000, 64, "fp32", causal=1, pre_ln=1, gelu_tanh=1, head=0)
SHAPES["fp32_postln_256"] = synthdata.ModelShape(2, 256, 4, 1024, 1000, 64, "fp32")
SHAPES["bf16_postln_256"] = synthdata.ModelShape(2, 256, 4, 1024, 1000, 64, "bf16")


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("cost_aware", [0, 1])
@pytest.mark.parametrize("collecting", [False, True])
def test_ratios_against_a_score(name, cost_aware, collecting):
    shape = SHAPES[name]
    m = mi.Mimose(synthdata.shape_dict(shape), 0, arena_bytes=256 * MiB, cost_aware=cost_aware)
    m.load_params(synthdata.make_params(shape, 11, perturb=True))
    if not collecting:
        m.force_plan(0)
    for seed, lengths in ((12, LENGTHS), (13, [max(LENGTHS)] * 3), (14, [40, 1, 1, 1, 1, 1]), (15, [48, 30, 9, 2, 14, 5, 20, 11] * 2)):
        tokens, labels, lens = synthdata.make_padded_batch(shape, lengths, seed)
        logp = m.score(tokens, labels, lens)
        for sign in (1.0, -1.0):
            # bounds of 0 hold back the gain of every ratio on the side that the advantage's sign rewards
            _, stats, _, _ = m.train_step_policy(tokens, labels, logp, np.full_like(logp, sign), ref_logp=logp, clip_low=0.0, clip_high=0.0,
                                                 kl_weight=0.1, lengths=lens)
            assert stats[1] == 0 and stats[2] == 0, (lengths, sign, stats)
    m.close()
