"""A captured pass over packed sequences, replayed with other lengths: the graph holds the buffers and how many sequences they hold at most, the
lengths lie on the device."""
import numpy as np
import pytest
import torch

from gpu_util import sync
from test_gpu_packed_attention import KEEP, Call

pytestmark = pytest.mark.gpu
NAMES = ("out", "lse", "dq", "dk", "dv")


def replays(dtype, h, hk, d, captured, others, causal):
    """Lengths may add up to fewer rows than the buffers have, and sequences may have none."""
    T = sum(captured)
    c = Call(dtype, h, hk, d, captured, seed=1)
    c.fwd(causal)
    c.bwd(causal)
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream().cuda_stream
        c.fwd(causal, stream=s)
        c.bwd(causal, stream=s)
    for i, lengths in enumerate(others):
        e = Call(dtype, h, hk, d, lengths, behind=T - sum(lengths), seed=2 + i)
        assert (e.T, e.n_seq) == (c.T, c.n_seq)
        for x in ("q", "k", "v", "do", "ends"):
            getattr(c, x).copy_(getattr(e, x))
        for x in NAMES:
            getattr(c, x).fill_(KEEP)
        sync()
        graph.replay()
        sync()
        e.check(causal)                                           # the eager pass against 64 bits, rows of no sequence included
        for x in NAMES:
            assert torch.equal(getattr(c, x), getattr(e, x)), (lengths, x)


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,h,hk,d", [(1, 4, 2, 64), (1, 4, 4, 32), (1, 3, 1, 128), (0, 4, 2, 64), (0, 2, 2, 128)])
def test_few_sequences(dtype, h, hk, d, causal):
    replays(dtype, h, hk, d, [90, 33, 130], [[10, 200, 43], [0, 253, 0], [1, 0, 64], [90, 33, 130], [0, 0, 0], [251, 1, 1]], causal)


@pytest.mark.parametrize("dtype,d", [(1, 64), (1, 128), (0, 32)])
def test_more_sequences_than_are_sorted(dtype, d):
    rng = np.random.default_rng(d)
    others = [rng.integers(0, 9, 70).tolist() for _ in range(3)]
    others[1][-1], others[2][0] = 200, 300                        # one long sequence, behind all others and before them
    assert all(sum(x) <= 70 * 10 for x in others)
    replays(dtype, 2, 1, d, [10] * 70, others, 1)


def test_one_that_fills_the_buffer():
    """Chosen for many short sequences, replayed with a single long one, and the other way round."""
    replays(1, 12, 12, 64, [64] * 12, [[0] * 11 + [768], [768] + [0] * 11, [1] * 12], 1)
    replays(1, 2, 1, 64, [1400], [[1], [1399], [0]], 1)
