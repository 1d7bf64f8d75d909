"""The oracle of the update with moments in 8 bits: its codes against torch's e4m3 type, its rounding and its drift."""
import numpy as np
import pytest
import torch

from oracle import optimizer8 as o8
from oracle.optimizer import AdamW


def test_codes_are_those_of_the_e4m3_type():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.tensor(codes).view(torch.float8_e4m3fn).double().numpy()
    got = o8.decode(codes)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])
    # the code of a code's own value is that code, whatever the dither (the block's largest value is 448, its scale 1)
    x = np.concatenate([got[:127], -got[1:127], [448.0]])
    c, s, _ = o8.encode(x, o8.K_M, 5)
    assert s[0] == 1.0 and np.array_equal(o8.decode(c), x)


def test_rounding_averages_out_over_the_updates():
    x = np.abs(np.random.default_rng(1).standard_normal(256)) + 1e-4
    mean = np.mean([o8.decode(c) * np.repeat(s, 256) for c, s, _ in (o8.encode(x, o8.K_V, t) for t in range(1, 1001))], axis=0)
    # a Weyl sequence of the golden ratio over N updates leaves a mean within 3 log2(N) / N codes of an eighth
    assert np.abs(mean / x - 1).max() < 3 * 10 / 1000 / 8 * 2


def test_a_slow_second_moment_follows_instead_of_standing_still():
    """1500 updates of unit gradients, beta2 = 0.999: the held root follows sqrt(1 - 0.999^t); rounded to the nearest
    code it would stop far below, where a code's half step is more than an update's."""
    n, t = 256, 1500
    rng = np.random.default_rng(2)
    v, vs = np.zeros(n, np.uint8), np.zeros(1)
    m, ms, p = np.zeros(n, np.uint8), np.zeros(1), np.zeros(n)
    size = np.exp(rng.standard_normal(n))
    size[0] = size.max() * 2
    for k in range(1, t + 1):
        r = o8.step(p, size * np.where(rng.random(n) < 0.5, -1, 1), m, v, ms, vs, k, 0.0, 0.9, 0.999, 1e-8, 0.0)
        m, v, ms, vs = r["m"], r["v"], r["m_scale"], r["v_scale"]
    want = size * np.sqrt(1 - 0.999 ** t)
    ratio = o8.decode(v) * vs[0] / want
    assert abs(np.mean(ratio) - 1) < 0.02 and np.abs(ratio - 1).max() < 0.2


@pytest.mark.parametrize("decay", [0.0, 0.1])
def test_first_update_is_that_of_the_plain_oracle(decay):
    rng = np.random.default_rng(3)
    p, g = rng.standard_normal((2, 300))
    h = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=decay)
    want = AdamW(**h).step({"w": p[None]}, {"w": g[None]})["w"][0]
    z = np.zeros(300, np.uint8)
    r = o8.step(p, g, z, z, np.zeros(2), np.zeros(2), 1, **h)
    assert np.abs(r["p"] - want).max() < 1e-15
    assert np.abs(o8.decode(r["m"]) * np.repeat(r["m_scale"], 256)[:300] / (0.1 * g) - 1).max() <= 0.125


def test_values_that_are_not_finite_are_nan_codes_outside_the_scale():
    x = np.array([1.0, np.inf, -np.inf, np.nan, -2.0])
    c, s, _ = o8.encode(x, o8.K_M, 1)
    assert s[0] == 2.0 / 448 and np.isnan(o8.decode(c)[1:4]).all() and o8.decode(c)[4] == -448
