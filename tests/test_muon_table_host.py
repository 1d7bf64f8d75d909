"""The list of matrices that MuonTable is made of, with stand-ins for tensors, streams and the library: no GPU."""
import contextlib

import pytest
import torch

import paper_2209_02478_amd as mi
from paper_2209_02478_amd import binding


class Tensor:
    """What MuonTable asks of a device tensor."""

    def __init__(self, *shape, dtype=torch.float32, device="cuda:0", contiguous=True):
        self.shape, self.dtype, self.device, self.contiguous = torch.Size(shape), dtype, torch.device(device), contiguous
        self.is_cuda = self.device.type == "cuda"

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 1 << 20


def entry(**other):
    return dict(dict(master=Tensor(30, 10), grad=Tensor(30, 10), momentum=Tensor(30, 10), lowp=Tensor(30, 10, dtype=torch.bfloat16)), **other)


@pytest.fixture
def calls(monkeypatch):
    """What the table does, in order: (call, the stream that torch has current at that time)."""
    log, current = [], [7]
    stream_of = lambda pointer: type("Stream", (), {"cuda_stream": pointer})()

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream.cuda_stream
        yield
        current[0] = before

    def empty(n, **kw):
        log.append(("memory", current[0]))
        return Tensor(n, dtype=torch.uint8)

    def table(entries, parts, memory, nbytes, stream):
        log.append(("copy", stream))
        return binding.mimose_muon_table()

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream_of(current[0]))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: stream_of(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda pointer, device=None: stream_of(pointer))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(binding, "mimose_op_muon_table_bytes", lambda entries, parts: 512)
    monkeypatch.setattr(binding, "mimose_op_muon_table", table)
    return log


@pytest.mark.parametrize("stream, used", [(None, 7), (7, 7), (9, 9), (0, 0)])
def test_memory_belongs_to_the_stream_that_fills_it(calls, stream, used):
    mi.MuonTable([entry()], stream=stream)
    assert calls == [("memory", used), ("copy", used), ("memory", used)]
    assert torch.cuda.current_stream().cuda_stream == 7


@pytest.mark.parametrize("name, tensor", [
    ("grad", Tensor(30, 10, device="cuda:1")), ("momentum", Tensor(30, 10, device="cpu")), ("lowp", Tensor(30, 10, dtype=torch.bfloat16, device="cuda:1")),
    ("grad", Tensor(10, 30)), ("grad", Tensor(300)), ("momentum", Tensor(30, 10, dtype=torch.bfloat16)), ("lowp", Tensor(30, 10)),
    ("master", Tensor(30, 10, dtype=torch.float64)), ("master", Tensor(300)), ("master", Tensor(3, 10, 10)), ("grad", Tensor(30, 10, contiguous=False)),
    ("momentum", None), ("grad", None)])
def test_tensors_that_are_refused(calls, name, tensor):
    with pytest.raises(ValueError, match=name):
        mi.MuonTable([entry(), entry(**{name: tensor})])
    assert not calls


def test_lists(calls):
    there = {k: Tensor(*t.shape, dtype=t.dtype, device="cuda:1") for k, t in entry().items()}
    with pytest.raises(ValueError, match="master"):
        mi.MuonTable([entry(), there])
    mi.MuonTable([there])
    mi.MuonTable([entry(lowp=None)])
    given = [entry()]
    assert mi.MuonTable(given).matrices == given                  # and so keeps them alive
