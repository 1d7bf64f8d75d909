"""The oracle of the losses on token log-probabilities against central differences, torch's autograd and closed forms."""
import numpy as np
import pytest
import torch

from oracle import token_loss as tl


def case(seed, T=12, V=17):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, V)) * 2
    labels = rng.integers(0, V, T)
    labels[[1, 7]] = -1
    labels[4] = V                                   # outside: left out as well
    return rng, x, labels


def differences(f, x, h=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        g[i] = (f(a) - f(b)) / (2 * h)
    return g


def test_logprob_of_a_uniform_row_and_of_masked_columns():
    x = np.zeros((2, 8))
    x[1, 3:] = -np.inf
    logp, soft = tl.token_logprob(x, np.array([5, 0]))
    assert np.allclose(logp, [-np.log(8), -np.log(3)], atol=1e-15)
    assert np.all(soft[1, 3:] == 0)


@pytest.mark.parametrize("smoothing", [0.0, 0.2])
def test_preference_gradient_against_differences(smoothing):
    rng, x, labels = case(1)
    ends, ref = [3, 3, 9, 12], rng.standard_normal(4) * 3      # (the second sequence has no rows)
    f = lambda y: tl.preference_loss(y, labels, ends, ref, 0.7, smoothing)["loss"]  # noqa: E731
    got = tl.preference_loss(x, labels, ends, ref, 0.7, smoothing)["dlogits"]
    # central differences: truncation h^2 / 6 times a third derivative of order 1, rounding 1e-16 / h
    assert np.abs(got - differences(f, x)).max() < 1e-9
    assert np.abs(got.sum(1)).max() < 1e-15 and not got[[1, 4, 7]].any()


@pytest.mark.parametrize("kl_weight", [0.0, 0.3])
def test_policy_gradient_against_differences(kl_weight):
    rng, x, labels = case(2)
    T = len(labels)
    old = tl.token_logprob(x, labels)[0] + rng.standard_normal(T) * 0.5
    ref = old + rng.standard_normal(T) * 0.4
    adv, weight = rng.standard_normal(T), rng.random(T)
    weight[5] = 0.0
    args = (labels, old, ref, adv, weight, 0.25, 0.2, 0.3, kl_weight)
    got = tl.policy_loss(x, *args)
    assert np.abs(got["dlogits"] - differences(lambda y: tl.policy_loss(y, *args)["stats"][0], x)).max() < 1e-9
    assert got["stats"][2] > 0 and not got["dlogits"][[1, 4, 5, 7]].any()


def test_losses_against_torch_autograd():
    rng, x, labels = case(3)
    ok = tl.scored_rows(labels, x.shape[1])
    ends, ref = [4, 6, 6, 12], rng.standard_normal(4)
    t = torch.tensor(x, requires_grad=True)
    rows = np.flatnonzero(ok)
    lp = torch.log_softmax(t, 1)[rows, labels[rows]]
    logp = torch.zeros(len(labels), dtype=torch.float64).index_put((torch.tensor(rows),), lp)
    seq = torch.stack([logp[a:b].sum() for a, b in zip([0] + ends[:-1], ends)])
    h = seq - torch.tensor(ref)
    loss = -torch.nn.functional.logsigmoid(0.3 * (h[0::2] - h[1::2])).mean()
    loss.backward()
    got = tl.preference_loss(x, labels, ends, ref, 0.3, 0.0)
    assert abs(got["loss"] - float(loss.detach())) < 1e-14
    assert np.abs(got["dlogits"] - t.grad.numpy()).max() < 1e-15
    # one step from the sampling policy, no KL: the plain policy gradient
    old = tl.token_logprob(x, labels)[0]
    adv = rng.standard_normal(len(labels))
    t = torch.tensor(x, requires_grad=True)
    (-(torch.log_softmax(t, 1)[rows, labels[rows]] * torch.tensor(adv[rows])).sum()).backward()
    got = tl.policy_loss(x, labels, old, None, adv, None, 1.0, 0.2, 0.2, 0.0)
    assert np.abs(got["dlogits"] - t.grad.numpy()).max() < 1e-14 and got["stats"][1] == got["stats"][2] == 0
