"""Fine-tuning a causal model with preferences and with a policy loss, under a memory budget.

    python examples/finetune.py [--model gpt2_medium] [--pairs 4] [--steps 12] [--state-bits 8]

One context plays both models in turn: before the first update it is the reference model and scores every batch
(`score`); after that it is trained, first on pairs of answers (`train_step_preference`), then on sampled tokens with
advantages (`train_step_policy`: the old policy's log-probabilities are scored at the start of each round, and two updates
are made from them).  The update holds its moments in 8 bits, which leaves 6 bytes a parameter more of the budget to
activations, so the planner rebuilds fewer layers.  Data and weights are random (there is nothing to learn but the batches
themselves): watch the losses fall on them.
"""
import argparse
import os
import sys

import numpy as np
import torch  # noqa: F401  (before the library is loaded: both then share one HIP runtime)

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import synthdata  # noqa: E402
import paper_2209_02478_amd as mi  # noqa: E402


def make_pairs(shape, pairs, length, seed):
    """A batch of 2 * pairs padded samples, answers behind a prompt of a quarter of the batch's length that a pair shares."""
    rng = np.random.default_rng(seed)
    prompt = max(1, length // 4)
    lengths = rng.integers(prompt + 2, length + 1, 2 * pairs).astype(np.int32)
    lengths[0] = length
    tokens, labels, lengths = synthdata.make_padded_batch(shape, lengths, seed)
    tokens[1::2, :prompt] = tokens[0::2, :prompt]
    labels[1::2, :prompt - 1] = labels[0::2, :prompt - 1]
    labels[:, :prompt - 1] = -1                        # the prompt is not scored
    return tokens, labels, lengths


def layers_rebuilt(plan):
    return bin(plan).count("1")


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--model", default="gpt2_medium", help="entry of synthdata.WORKLOADS")
    ap.add_argument("--pairs", type=int, default=4)
    ap.add_argument("--steps", type=int, default=12, help="updates of each kind")
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--lr", type=float, default=2e-5)
    ap.add_argument("--budget-frac", type=float, default=0.6, help="of what the longest batch needs without checkpointing")
    a = ap.parse_args(argv)
    work = synthdata.WORKLOADS[a.model]
    shape, d = work.shape, synthdata.shape_dict(work.shape)
    hyper = dict(lr=a.lr, beta1=0.9, beta2=0.95, weight_decay=0.0)

    def no_checkpoint_peak(bits):
        cal = mi.Mimose(d, 0, device=None)
        cal.optimizer_init(state_bits=bits, **hyper)
        cal.force_plan(0)
        peak, _ = cal.dry_step(2 * a.pairs, shape.max_seq)
        cal.close()
        return peak

    budget = int(no_checkpoint_peak(32) * a.budget_frac)
    m = mi.Mimose(d, budget)
    m.load_params(synthdata.make_params(shape, work.seed))
    m.optimizer_init(state_bits=a.state_bits, **hyper)
    print(f"{a.model}: budget {budget >> 20} MiB, fixed {m.stats()['fixed_bytes'] >> 20} MiB with {a.state_bits}-bit moments", flush=True)

    # three batches of different lengths; the reference model's sums are scored once
    batches = [make_pairs(shape, a.pairs, max(16, shape.max_seq * k // 4), 100 + k) for k in (1, 2, 3)]
    refs = [m.score(t, y, n) for t, y, n in batches]
    first, last = {}, {}
    for step in range(a.steps):
        k = step % len(batches)
        tokens, labels, lengths = batches[k]
        loss, margin, peak, plan = m.train_step_preference(tokens, labels, refs[k].sum(1), beta=0.1, lengths=lengths)
        m.optimizer_step()
        first.setdefault(k, loss)
        last[k] = loss
        print(f"preference {step}: length {tokens.shape[1]}, loss {loss:.4f}, preferred in {(margin > 0).mean():.0%}, "
              f"peak {peak >> 20} MiB, {layers_rebuilt(plan)} layers rebuilt", flush=True)
    preference = {k: (first[k], last[k]) for k in first}

    policy = []
    rng = np.random.default_rng(7)
    advantages = [np.repeat(rng.standard_normal((t.shape[0], 1)), t.shape[1], 1).astype(np.float32) for t, _, _ in batches]
    for step in range(a.steps):
        k = step // 2 % len(batches)
        tokens, labels, lengths = batches[k]
        if step % 2 == 0:
            old = m.score(tokens, labels, lengths)     # what the tokens' policy was before these two updates
        loss, stats, peak, plan = m.train_step_policy(tokens, labels, old, advantages[k], ref_logp=refs[k], kl_weight=0.02,
                                                      clip_high=0.28, lengths=lengths)
        m.optimizer_step()
        policy.append((loss, float(stats[1]), float(stats[2])))
        print(f"policy {step}: loss {loss:.4f}, KL {stats[1]:.4f}, clipped {stats[2]:.2%}, peak {peak >> 20} MiB, "
              f"{layers_rebuilt(plan)} layers rebuilt", flush=True)
    peak = m.stats()["peak_bytes_max"]
    m.close()
    return dict(budget=budget, peak=peak, preference=preference, policy=policy)


if __name__ == "__main__":
    main()
