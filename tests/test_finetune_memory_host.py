"""What an iteration takes of the arena does not depend on its loss: a dry step's peak, a plan and the planner's samples hold for the
preference and the policy loss as for the cross-entropy.  libmimose on the stand-in for the HIP runtime of test_launch_errors: host
memory, kernels that are not run."""
import pytest

from test_launch_choice import run
from test_launch_errors import runtime  # noqa: F401

SETUP = """
    import synthdata
    dtype, pre_ln, head, H = sys.argv[2], *map(int, sys.argv[3:6])
    shape = synthdata.ModelShape(3, H, H // 32, 2 * H, 64, 96, dtype, causal=pre_ln, pre_ln=pre_ln, head=head)
    cfg = lambda **kw: mi.make_cfg(synthdata.shape_dict(shape), **kw)
    def context(budget, **kw):
        global memory
        memory = np.zeros(budget + 512, np.uint8)
        return mi.mimose_init(cfg(**kw), budget, (memory.ctypes.data + 255) // 256 * 256, budget)
    def steps(ctx, B, L, lengths):
        # every loss, as functions that return the peak
        tokens, labels = synthdata.make_batch(shape, B, L, 3)
        z, s = np.zeros((B, L), np.float32), np.zeros(B, np.float32)
        n = None if lengths is None else np.array(lengths, np.int32)
        yield "cross-entropy", lambda: (mi.mimose_train_step(ctx, tokens, labels) if n is None else mi.mimose_train_step_padded(ctx, tokens, labels, n))[1]
        if B % 2 == 0:
            yield "preference", lambda: mi.mimose_train_step_preference(ctx, tokens, labels, s, lengths=n)[2]
        for ref in (None, z):
            for weight in (None, z):
                yield "policy", lambda: mi.mimose_train_step_policy(ctx, tokens, labels, z, z, ref_logp=ref, weight=weight, lengths=n)[2]
"""
MODELS = [("bf16", 1, 0, 32), ("bf16", 0, 1, 32), ("bf16", 0, 0, 64), ("fp32", 1, 0, 32), ("fp32", 0, 1, 64), ("bf16", 1, 1, 256)]


@pytest.mark.parametrize("model", MODELS)
def test_a_budget_of_the_dry_peak(runtime, model):  # noqa: F811
    run(runtime, SETUP + """
    for B, L, lengths in ((2, 1, None), (1, 1, None), (6, 33, None), (6, 33, [33, 20, 7, 33, 1, 30]), (16, 96, None), (16, 96, [96, 2] * 8),
                          (96, 1, None), (2, 96, [96, 1])):
        for plan in (0, 0b111, 0b010):
            ctx = context(64 << 20)
            mi.mimose_force_plan(ctx, plan)
            want, _ = mi.mimose_dry_step(ctx, B, L)
            mi.mimose_destroy(ctx)
            ctx = context(want)
            mi.mimose_force_plan(ctx, plan)
            for name, step in steps(ctx, B, L, lengths):
                got = step()
                assert got == want, (name, B, L, lengths, plan, got - want)
            mi.mimose_destroy(ctx)
    """, *model)


@pytest.mark.parametrize("model", MODELS[:3])
def test_a_planner_that_collected_on_another_loss(runtime, model):  # noqa: F811
    """A budget that makes it drop layers; iterations of every loss after one loss's samples: no plan is made anew."""
    run(runtime, SETUP + """
    host = mi.mimose_init(cfg(), 0, None, 0)
    mi.mimose_force_plan(host, 0)
    budget = int(0.97 * mi.mimose_dry_step(host, 8, 96)[0])
    predicted = {}
    for first in range(6):
        ctx = context(budget, sheltered_steps=4)
        for L in (16, 40, 64, 90):
            list(steps(ctx, 8, L, None))[first][1]()
        for L in (96, 95, 94, 93, 92):
            peaks = {step() for _, step in steps(ctx, 8, L, None)}
            assert len(peaks) == 1 and max(peaks) <= budget, (first, L, peaks)
            guess = mi.mimose_get_stats(ctx)["predicted_peak_last"]
            assert guess >= max(peaks) and predicted.setdefault(L, guess) == guess, (first, L, guess, peaks)
        assert mi.mimose_get_stats(ctx)["replans"] == 0
        mi.mimose_destroy(ctx)
    """, *model)
