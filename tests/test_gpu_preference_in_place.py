"""A preference loss with its gradient in place has the bits that it has beside the logits, on either side of the sizes at which either
form goes past the caches, on rows of any alignment."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, TDT
from test_gpu_token_loss import run_preference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,V,ld,offset", [(1, 50257, 50304, 0), (1, 50257, 50257, 3), (0, 30522, 30528, 0)])
@pytest.mark.parametrize("pairs", [2, 9])
@pytest.mark.parametrize("mb", [20, 159.9, 160.1, 300, 639.9, 640.1])
def test_bits(dtype, V, ld, offset, pairs, mb):
    T = round(mb * 2 ** 20 / (ld * (2 if dtype else 4)))
    g = torch.Generator(device=DEV).manual_seed(T)
    buf = torch.randn(T * ld + 8, generator=g, device=DEV, dtype=torch.float32).mul_(2).to(TDT[dtype])
    logits = buf[offset:offset + T * ld].view(T, ld)
    labels = np.random.default_rng(T).integers(0, V, T).astype(np.int32)
    labels[T // 3:T // 2] = -1
    ends = [T * (k + 1) // (2 * pairs) for k in range(2 * pairs)]
    ref = np.full(2 * pairs, -np.log(V) * T / (2 * pairs), np.float32)
    d = torch.full((T, ld), 9.0, dtype=TDT[dtype], device=DEV)
    beside = run_preference(dtype, logits, ld, labels, ends, pairs, 0, ref, 0.01, 0.1, d, T, V)
    inside = run_preference(dtype, logits, ld, labels, ends, pairs, 0, ref, 0.01, 0.1, logits, T, V)
    assert all(torch.equal(beside[k], inside[k]) for k in beside)
    assert torch.isfinite(d).all() and d[:T // 3, :V].any(1).all() and not d[T // 3:T // 2].any() and not d[:, V:].any()
    assert torch.equal(d, logits)
