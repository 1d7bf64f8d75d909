"""A table whose memory, copy and updates are on a stream of their own."""
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, sync

pytestmark = pytest.mark.gpu


def entry(n, bits):
    gen = torch.Generator().manual_seed(n)
    dt = torch.uint8 if bits == 8 else torch.float32
    t = dict(master=torch.randn(n, generator=gen), grad=torch.randn(n, generator=gen), m=torch.zeros(n, dtype=dt), v=torch.zeros(n, dtype=dt),
             decay=1)
    if bits == 8:
        t.update(m_scale=torch.zeros(-(-n // 256)), v_scale=torch.zeros(-(-n // 256)))
    return {k: v.to(DEV) if torch.is_tensor(v) else v for k, v in t.items()}


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("where", ["current", "own", "default"])
def test_streams(bits, where):
    a, b = entry(70001, bits), entry(70001, bits)
    ta = mi.AdamWTable([a], bits)
    sync()
    mi.mimose_op_adamw_step(ta, 1)
    sync()
    own = torch.cuda.Stream()
    stream = {"current": None, "own": own.cuda_stream, "default": torch.cuda.default_stream().cuda_stream}[where]
    tb = mi.AdamWTable([b], bits, stream=stream)
    mi.mimose_op_adamw_step(tb, 1, stream=stream)
    sync()
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    for k in ("master", "m", "v"):
        assert torch.equal(a[k], b[k]), k
