"""The list of tensors that AdamWTable is made of, with stand-ins for tensors, streams and the library: no GPU."""
import contextlib

import pytest
import torch

import paper_2209_02478_amd as mi
from paper_2209_02478_amd import binding


class Tensor:
    """What AdamWTable asks of a device tensor."""
    is_cuda = True

    def __init__(self, n, dtype=torch.float32, device="cuda:0"):
        self.n, self.dtype, self.device = n, dtype, torch.device(device)

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def entry(**other):
    t = dict(master=Tensor(300), grad=Tensor(300), m=Tensor(300, torch.uint8), v=Tensor(300, torch.uint8), m_scale=Tensor(2), v_scale=Tensor(2),
             lowp=Tensor(300, torch.bfloat16))
    return dict(t, **other)


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
        return Tensor(n, torch.uint8)

    def table(entries, bits, memory, nbytes, stream):
        log.append(("copy", stream))
        return binding.mimose_adamw_table()

    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: stream_of(current[0]))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: stream_of(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda pointer, device=None: stream_of(pointer))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(binding, "mimose_op_adamw_table_bytes", lambda entries, bits: 512)
    monkeypatch.setattr(binding, "mimose_op_adamw_table", table)
    return log


@pytest.mark.parametrize("stream, used", [(None, 7), (7, 7), (9, 9), (0, 0)])
def test_memory_belongs_to_the_stream_that_fills_it(calls, stream, used):
    # taken from another stream's memory, it could still be read or written there by what was queued before
    mi.AdamWTable([entry()], 8, stream=stream)
    assert calls == [("memory", used), ("copy", used)]
    assert torch.cuda.current_stream().cuda_stream == 7


@pytest.mark.parametrize("name, tensor", [("grad", Tensor(300, device="cuda:1")), ("m", Tensor(300, torch.uint8, "cuda:1")),
                                          ("v_scale", Tensor(2, device="cuda:1")), ("lowp", Tensor(300, torch.bfloat16, "cuda:1"))])
def test_tensors_of_several_devices(calls, name, tensor):
    with pytest.raises(ValueError, match=name):
        mi.AdamWTable([entry(), entry(**{name: tensor})], 8)
    assert not calls


def test_lists_of_several_devices(calls):
    there = {k: Tensor(t.n, t.dtype, "cuda:1") for k, t in entry().items()}
    with pytest.raises(ValueError, match="master"):
        mi.AdamWTable([entry(), there], 8)
    mi.AdamWTable([there], 8)
