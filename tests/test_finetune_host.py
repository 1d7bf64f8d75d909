"""The executor's fine-tuning calls without a GPU: memory of the update's state, and what host-only contexts refuse."""
import numpy as np
import pytest

import synthdata
import paper_2209_02478_amd as mi


def shape(dtype):
    return synthdata.ModelShape(3, 128, 2, 512, 1003, 96, dtype, causal=1, pre_ln=1, gelu_tanh=1, head=0)


def context(dtype, budget=0):
    return mi.Mimose(synthdata.shape_dict(shape(dtype)), budget, device=None)


def up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("bits", [8, 32])
def test_fixed_bytes_of_the_state(dtype, bits):
    """Moments (and scales) of every tensor, the master of a bf16 model, and the tables, each on 256 bytes; peaks rise by them."""
    plain, m = context(dtype), context(dtype)
    m.optimizer_init(state_bits=bits)
    want, chunks = 0, 0
    for s in m.shapes.values():
        n = int(np.prod(s))
        want += 2 * up(n if bits == 8 else 4 * n) + (up(4 * n) if dtype == "bf16" else 0)
        want += 2 * up(4 * (-(-n // 256))) if bits == 8 else 0
        chunks += -(-n // 16384)
    want += up((72 if bits == 8 else 56) * len(m.shapes)) + up(16 * chunks)
    assert m.stats()["fixed_bytes"] - plain.stats()["fixed_bytes"] == want
    for plan in (0, 0b101):
        for c in (plain, m):
            c.force_plan(plan)
        assert m.dry_step(4, 33)[0] - plain.dry_step(4, 33)[0] == want
    plain.close()
    m.close()


def test_a_budget_for_8_bits_and_not_for_32():
    plain = context("bf16")
    fixed, n = plain.stats()["fixed_bytes"], sum(int(np.prod(s)) for s in plain.shapes.values())
    plain.close()
    budget = fixed + 8 * n
    m = context("bf16", budget)
    with pytest.raises(mi.MimoseError) as e:
        m.optimizer_init()
    assert e.value.code == mi.MIMOSE_ERR_OOM_BUDGET and m.stats()["fixed_bytes"] == fixed
    m.optimizer_init(state_bits=8)
    assert fixed + 6 * n <= m.stats()["fixed_bytes"] <= budget
    with pytest.raises(mi.MimoseError) as e:
        m.optimizer_init(state_bits=8)
    assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG and "already" in str(e.value)
    m.close()


def test_host_only_contexts_refuse():
    m = context("fp32")
    tokens, labels = synthdata.make_batch(shape("fp32"), 4, 9, 1)
    z = np.zeros((4, 9), np.float32)
    for call in (lambda: m.score(tokens, labels), lambda: m.train_step_preference(tokens, labels, z[:, 0]),
                 lambda: m.train_step_policy(tokens, labels, z, z)):
        with pytest.raises(mi.MimoseError) as e:
            call()
        assert e.value.code == mi.MIMOSE_ERR_NOT_READY
    for bits in (0, 4, 16, 64):
        with pytest.raises(mi.MimoseError) as e:
            m.optimizer_init(state_bits=bits)
        assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG
    m.dry_step(4, 9)
    with pytest.raises(mi.MimoseError) as e:
        m.optimizer_init(state_bits=8)
    assert e.value.code == mi.MIMOSE_ERR_NOT_READY
    m.close()
