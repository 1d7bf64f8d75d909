"""The 64-bit form of packed attention against torch's autograd over a plain masked softmax."""
import numpy as np
import pytest
import torch

from oracle import packed_attention as oa


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("h,hk", [(2, 2), (6, 2), (3, 1)])
def test_definition(h, hk, causal):
    rng = np.random.default_rng(h)
    ends, d, T, scale = [4, 4, 5, 17], 8, 17, 0.4
    q, k, v, do = (rng.standard_normal((T, n, d)) for n in (h, hk, hk, h))
    tq, tk, tv = (torch.tensor(x, requires_grad=True) for x in (q, k, v))
    seq = torch.searchsorted(torch.tensor(ends), torch.arange(T), right=True)
    seen = seq[:, None] == seq[None, :]
    if causal:
        seen = seen & torch.ones(T, T, dtype=torch.bool).tril()
    ek, ev = (x.repeat_interleave(h // hk, 1) for x in (tk, tv))
    s = (torch.einsum("ihd,jhd->hij", tq, ek) * scale).masked_fill(~seen, -torch.inf)
    out = torch.einsum("hij,jhd->ihd", torch.softmax(s, 2), ev)
    (out * torch.tensor(do)).sum().backward()
    got, lse, out_off, lse_off = oa.forward(q, k, v, ends, scale, causal, 2.0 ** -8)
    assert np.allclose(got, out.detach().numpy(), rtol=0, atol=1e-13)
    assert np.allclose(lse, torch.logsumexp(s, 2).detach().numpy(), rtol=0, atol=1e-13)
    grads = oa.backward(q, k, v, got, lse, do, ends, scale, causal, 2.0 ** -8)
    for g, t in zip(grads, (tq, tk, tv)):
        assert np.allclose(g, t.grad.numpy(), rtol=0, atol=1e-12)
    assert (out_off > 0).all() and (lse_off > 0).all() and all((o > 0).all() for o in grads[3:])
