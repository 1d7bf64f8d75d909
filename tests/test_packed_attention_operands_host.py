"""Tensors that packed attention refuses before it takes their addresses, with stand-ins for device tensors: nothing is launched."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from paper_2209_02478_amd import binding

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Tensor:
    """What the calls ask of a device tensor."""

    def __init__(self, at, dtype, *shape, device=0, contiguous=True):
        self.at, self.dtype, self.shape, self.device_id, self.contiguous = at, dtype, shape, device, contiguous
        self.is_cuda = device >= 0

    def get_device(self):
        return self.device_id

    def is_contiguous(self):
        return self.contiguous

    def numel(self):
        return int(np.prod(self.shape))

    def data_ptr(self):
        return self.at


def operands(dtype=BF16, **other):
    at = [1 << k for k in range(30, 44)]
    rows = {name: Tensor(at[i], dtype, 10, w) for i, (name, w) in enumerate((("q", 256), ("k", 128), ("v", 128), ("out", 256), ("dout", 256), ("dq", 256),
                                                                             ("dk", 128), ("dv", 128)))}
    return dict(rows, lse=Tensor(at[8], F32, 4, 10), ends=Tensor(at[9], I32, 2), workspace=Tensor(at[10], torch.uint8, 1 << 12)) | other


def call(which, t, dtype=1, **other):
    a = dict(dtype=dtype, q=t["q"], ldq=256, k=t["k"], ldk=128, v=t["v"], ldv=128, out=t["out"], ldo=256, lse=t["lse"], ends=t["ends"], n_seq=2,
             T=10, n_heads=4, n_kv_heads=2, head_dim=64, causal=1, scale=0.125)
    if which == "bwd":
        a |= dict(dout=t["dout"], lddo=256, dq=t["dq"], lddq=256, dk=t["dk"], lddk=128, dv=t["dv"], lddv=128, workspace=t["workspace"], workspace_bytes=1 << 12)
    getattr(mi, "mimose_op_packed_attention_" + which)(**(a | other))


@pytest.fixture
def launched(monkeypatch):
    """Addresses that reached the library, which is a stand-in too."""
    log = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: log.append(a) or 0

    monkeypatch.setattr(binding, "load_library", lambda: Library())
    return log


WHICH = pytest.mark.parametrize("which", ["fwd", "bwd"])
ROWS = ["q", "k", "v", "out"]


def refused(launched, which, t, why, **other):
    for first in (False, True):                       # also where nothing has been looked at before
        if first:
            binding._TYPES.clear()
        with pytest.raises(mi.MimoseError, match=why) as e:
            call(which, t, **other)
        assert e.value.code == mi.MIMOSE_ERR_INVALID_ARG and which in str(e.value) and not launched


@WHICH
@pytest.mark.parametrize("name", ROWS + ["lse", "ends", "dout", "dq", "dk", "dv", "workspace"])
def test_off_the_device(launched, which, name):
    if which == "fwd" and name not in ROWS + ["lse", "ends"]:
        return
    x = operands()[name]
    refused(launched, which, operands(**{name: Tensor(x.at, x.dtype, *x.shape, device=-1)}), f"{name} is not on the device")
    refused(launched, which, operands(**{name: Tensor(x.at, x.dtype, *x.shape, device=1)}), "another device")
    refused(launched, which, operands(**{name: np.zeros(x.shape, np.float32)}), f"{name} is not on the device")


@WHICH
@pytest.mark.parametrize("name,wrong", [(n, w) for n in ROWS + ["dout", "dq", "dk", "dv"] for w in (F32, torch.float16)] +
                         [("lse", BF16), ("lse", torch.float64), ("ends", torch.int64), ("ends", F32)])
def test_types(launched, which, name, wrong):
    if which == "fwd" and name not in ROWS + ["lse", "ends"]:
        return
    x = operands()[name]
    refused(launched, which, operands(**{name: Tensor(x.at, wrong, *x.shape)}), f"{name} must be of")


@WHICH
def test_types_of_fp32(launched, which):
    refused(launched, which, operands(), "q must be of", dtype=0)
    call(which, operands(dtype=F32), dtype=0)


@WHICH
def test_gaps_and_counts(launched, which):
    for name in ("lse", "ends") + (("workspace",) if which == "bwd" else ()):
        x = operands()[name]
        refused(launched, which, operands(**{name: Tensor(x.at, x.dtype, *x.shape, contiguous=False)}), f"{name} must be contiguous")
    refused(launched, which, operands(ends=Tensor(1 << 39, I32, 1)), "fewer than 2")
    refused(launched, which, operands(), "too many", T=(1 << 32) + 10)
    refused(launched, which, operands(ends=Tensor(1 << 39, I32, 1 << 33)), "too many", n_seq=(1 << 32) + 2)
    refused(launched, which, {k: x.data_ptr() for k, x in operands().items()}, "too many", T=(1 << 32) + 10)


@WHICH
def test_what_is_taken(launched, which):
    """Tensors that are right, rows with leading dimensions of their own, and addresses, of all operands or of some."""
    t = operands()
    at = {k: x.data_ptr() for k, x in t.items()}
    some = dict(t, ends=at["ends"], workspace=at["workspace"], dk=at["dk"])
    strided = dict(t, q=Tensor(at["q"], BF16, 10, 256, contiguous=False), dv=Tensor(at["dv"], BF16, 10, 128, contiguous=False))
    binding._TYPES.clear()
    for given in (t, t, at, some, strided):
        call(which, given)
    assert len(launched) == 5 and all(a == launched[0] for a in launched)
    names = ("q", "k", "v", "out", "lse", "ends") if which == "fwd" else tuple(t)
    assert set(at[n] for n in names) <= set(launched[0])
