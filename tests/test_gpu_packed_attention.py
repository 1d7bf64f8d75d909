"""Attention over packed sequences with grouped heads, forward and backward, against its definition in 64 bits.  Bounds are
those of oracle/packed_attention.py: fp32 sums, and one rounding to the storage type of each probability and score gradient."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, TDT, sync
from oracle import packed_attention as oa

pytestmark = pytest.mark.gpu
UNIT = {0: 2.0 ** -24, 1: 2.0 ** -8}
KEEP = 7.0                                       # what outputs hold before a call


class Call:
    """Operands as a program holds them: q, k and v beside each other in rows of one buffer, gradients likewise."""

    def __init__(self, dtype, h, hk, d, lengths, behind=0, seed=0, pad=0, spread=1.0, separate=False, scale=None):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.h, self.hk, self.d = dtype, h, hk, d
        self.ends_host = list(np.cumsum(lengths)) if len(lengths) else []
        self.n_seq = len(lengths)
        self.rows = int(self.ends_host[-1]) if lengths else 0
        self.T = T = self.rows + behind
        self.scale = scale or 1.0 / d ** 0.5
        w = h + 2 * hk
        x = torch.randn(T, w, d, generator=g) * torch.tensor([spread] * (h + hk) + [1.0] * hk)[:, None]
        x[self.rows:] = float("nan")                              # rows of no sequence may hold anything
        x = x.to(TDT[dtype])
        self.values = [x[:, a:b].double().numpy() for a, b in ((0, h), (h, h + hk), (h + hk, w))]
        do = torch.randn(T, h, d, generator=g).to(TDT[dtype])
        do[self.rows:] = float("nan")
        self.do_value = do.double().numpy()
        if separate:                                              # each with a leading dimension of its own
            self.q, self.k, self.v = (self.place(x[:, a:b], p) for a, b, p in ((0, h, 16), (h, h + hk, 0), (h + hk, w, 8)))
            self.dq, self.dk, self.dv = (self.room(n, p) for n, p in ((h, 0), (hk, 24), (hk, 8)))
        else:
            buf, dbuf = self.place(x, pad), self.room(w, pad)
            cut = lambda b: [b[:, a * d:e * d] for a, e in ((0, h), (h, h + hk), (h + hk, w))]  # noqa: E731
            self.q, self.k, self.v = cut(buf)
            self.dq, self.dk, self.dv = cut(dbuf)
        self.do = self.place(do, pad)
        self.out, self.lse = self.room(h, pad), torch.full((h, T), KEEP, device=DEV)
        self.ends = torch.tensor(self.ends_host, dtype=torch.int32, device=DEV)
        self.ws = torch.full((max(16, mi.mimose_op_packed_attention_bwd_workspace_bytes(T, h, hk, d)),), 0xFF, dtype=torch.uint8, device=DEV)

    def place(self, x, pad):
        b = torch.full((x.shape[0], x.shape[1] * x.shape[2] + pad), float("nan"), dtype=TDT[self.dtype], device=DEV)
        b[:, :x.shape[1] * x.shape[2]] = x.flatten(1).to(DEV)
        return b[:, :x.shape[1] * x.shape[2]]

    def room(self, heads, pad):
        return torch.full((self.T, heads * self.d + pad), KEEP, dtype=TDT[self.dtype], device=DEV)[:, :heads * self.d]

    def heads(self, causal):
        return self.ends, self.n_seq, self.T, self.h, self.hk, self.d, int(causal), self.scale

    def fwd(self, causal, stream=None):
        a = [z for x in (self.q, self.k, self.v, self.out) for z in (x, x.stride(0))]
        mi.mimose_op_packed_attention_fwd(self.dtype, *a, self.lse, *self.heads(causal), stream=stream)

    def bwd(self, causal, stream=None):
        a = [z for x in (self.q, self.k, self.v, self.out) for z in (x, x.stride(0))]
        b = [z for x in (self.do, self.dq, self.dk, self.dv) for z in (x, x.stride(0))]
        mi.mimose_op_packed_attention_bwd(self.dtype, *a, self.lse, *b, *self.heads(causal), workspace=self.ws,
                                          workspace_bytes=self.ws.numel(), stream=stream)

    def split(self, x):
        return x.double().cpu().numpy().reshape(self.T, -1, self.d)

    def check(self, causal, backward=True):
        u, R = UNIT[self.dtype], self.rows
        q, k, v = (x[:R] for x in self.values)
        self.fwd(causal)
        sync()
        out, lse, out_off, lse_off = oa.forward(q, k, v, self.ends_host, self.scale, causal, u)
        within(self.split(self.out)[:R], out, out_off, "out")
        got = self.lse.double().cpu().numpy()
        within(got[:, :R], lse, lse_off, "lse")
        assert (self.split(self.out)[R:] == KEEP).all() and (got[:, R:] == KEEP).all()
        if not backward:
            return
        self.bwd(causal)
        sync()
        want = oa.backward(q, k, v, self.split(self.out)[:R], got[:, :R], self.do_value[:R], self.ends_host, self.scale, causal, u)
        for x, ref, off, name in zip((self.dq, self.dk, self.dv), want[:3], want[3:], ("dq", "dk", "dv")):
            within(self.split(x)[:R], ref, off, name)
            assert (self.split(x)[R:] == KEEP).all(), name


def within(got, ref, off, name):
    assert np.isfinite(got).all(), name
    bad = np.abs(got - ref) > off + 1e-37
    assert not bad.any(), (name, int(bad.sum()), float((np.abs(got - ref) / (off + 1e-37)).max()), np.argwhere(bad)[:3].tolist())


LENGTHS = [[1], [2], [17], [700, 1, 0, 65, 333], [0, 1, 0, 3, 0], [31, 32, 33], [63, 64, 65], [127, 128, 129, 1], [300], [5] * 9 + [200, 0, 77]]


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda x: "-".join(map(str, x))[:20])
@pytest.mark.parametrize("h,hk,d", [(4, 2, 64), (2, 2, 32), (3, 1, 128)])
@pytest.mark.parametrize("dtype", [1, 0])
def test_lengths(dtype, h, hk, d, lengths, causal):
    Call(dtype, h, hk, d, lengths, behind=len(lengths) % 3, seed=sum(lengths)).check(causal)


# backward passes of one launch and of two, and each way in which blocks share out the keys
WAYS = [(1, 12, 12, 64, [70] * 24), (1, 12, 12, 32, [40] * 40), (1, 8, 2, 64, [190]), (1, 6, 6, 64, [190, 3]), (1, 8, 2, 32, [200, 129]), (1, 2, 1, 128, [65, 140]),
        (1, 8, 2, 128, [190, 1]), (1, 6, 6, 128, [300]), (0, 12, 12, 64, [33] * 28), (0, 16, 16, 32, [33] * 64), (0, 8, 8, 128, [33] * 20), (0, 2, 1, 128, [400, 31]),
        (0, 4, 4, 64, [500, 0, 65]), (0, 12, 12, 64, [33] * 40), (0, 12, 12, 64, [33] * 50), (0, 8, 8, 128, [33] * 32), (0, 8, 8, 128, [33] * 42),
        (0, 8, 2, 128, [200] * 8), (0, 8, 2, 64, [200] * 9), (0, 16, 4, 32, [150] * 9), (1, 2, 1, 64, [700]),
        (1, 4, 2, 128, [650, 700]), (1, 2, 2, 32, [1000]), (1, 1, 1, 64, [641, 640])]


@pytest.mark.parametrize("causal", [1, 0])
@pytest.mark.parametrize("dtype,h,hk,d,lengths", WAYS, ids=[f"{x[0]}-{x[1]}-{x[2]}-{x[3]}-{len(x[4])}x{x[4][0]}" for x in WAYS])
def test_ways(dtype, h, hk, d, lengths, causal):
    Call(dtype, h, hk, d, lengths, behind=2, seed=d + len(lengths)).check(causal)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("h,hk", [(1, 1), (8, 1), (6, 6), (12, 4), (10, 5), (9, 3)])
def test_heads(dtype, h, hk):
    Call(dtype, h, hk, 64, [70, 3, 129], seed=h).check(1)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_leading_dimensions(dtype, d):
    Call(dtype, 4, 2, d, [65, 140], behind=3, pad=8, seed=1).check(1)
    Call(dtype, 4, 2, d, [65, 140], behind=3, separate=True, seed=2).check(0)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("count", [64, 65, 130, 4097])
def test_many_sequences(dtype, count):
    rng = np.random.default_rng(count)
    lengths = rng.integers(0, 4, count).tolist()
    lengths[count // 2], lengths[-1] = 150, 40
    Call(dtype, 2, 1, 32, lengths, behind=5, seed=count).check(1)


@pytest.mark.parametrize("dtype,d,causal", [(1, 32, 0), (1, 64, 0), (1, 64, 1), (1, 128, 1), (0, 64, 1)])
@pytest.mark.parametrize("count", [60, 70])
def test_blocks_for_the_whole_device(dtype, d, causal, count):
    """Heads of keys and rows enough to fill the device with blocks that share nothing, sequences in order of work and not."""
    rng = np.random.default_rng(d)
    lengths = rng.integers(1, 260, count).tolist()
    Call(dtype, 16, 16, d, lengths, behind=1, seed=d).check(causal)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("spread", [1e-20, 8.0])
def test_scores_of_any_size(dtype, spread):
    """No scores to tell apart, and scores so far apart that nearly every probability is zero."""
    Call(dtype, 2, 1, 64, [130, 40], spread=spread, seed=3).check(1)
    Call(dtype, 2, 1, 64, [130, 40], spread=spread, scale=0.7, seed=4).check(0)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("d", [64, 128])
def test_a_long_sequence(dtype, d):
    Call(dtype, 1, 1, d, [1500, 9], seed=5).check(1)


@pytest.mark.parametrize("dtype", [1, 0])
@pytest.mark.parametrize("causal", [0, 1])
def test_what_another_sequence_holds(dtype, causal):
    """Rows of infinities and NaN in one sequence, nothing of which reaches those before and behind it."""
    c = Call(dtype, 2, 1, 64, [40, 30, 50], seed=6)
    clean = Call(dtype, 2, 1, 64, [40, 30, 50], seed=6)
    for x in (c.q, c.k, c.v, c.do):
        x[40:70:2] = float("nan")
        x[41:70:2] = float("inf")
    for y in (c, clean):
        y.fwd(causal)
        y.bwd(causal)
    sync()
    for name in ("out", "dq", "dk", "dv"):
        a, b = getattr(c, name), getattr(clean, name)
        for rows in (slice(0, 40), slice(70, 120)):
            assert torch.equal(a[rows], b[rows]), name
    assert torch.equal(c.lse[:, :40], clean.lse[:, :40]) and torch.equal(c.lse[:, 70:], clean.lse[:, 70:])


@pytest.mark.parametrize("dtype", [1, 0])
def test_the_same_rows_whatever_lies_beside_them(dtype):
    """A sequence's results do not depend on where it lies, and are the same bit for bit each time."""
    a = Call(dtype, 4, 2, 64, [200], seed=7)
    b = Call(dtype, 4, 2, 64, [77, 200, 3], seed=8)
    for x, y in ((b.q, a.q), (b.k, a.k), (b.v, a.v), (b.do, a.do)):
        x[77:277] = y
    for c in (a, b, b):
        c.fwd(1)
        c.bwd(1)
    sync()
    for name in ("out", "dq", "dk", "dv"):
        assert torch.equal(getattr(b, name)[77:277], getattr(a, name)), name


def test_gradient_against_differences():
    """The kernel's gradient along a direction against central differences of the definition: h^2 of a third derivative, and
    the fp32 gradient's own bound."""
    c = Call(0, 2, 1, 32, [9, 33], seed=9)
    c.fwd(1)
    c.bwd(1)
    sync()
    rng = np.random.default_rng(1)
    q, k, v = c.values
    step = 1e-4
    for at, grad in enumerate((c.dq, c.dk, c.dv)):
        way = rng.standard_normal(c.values[at].shape)

        def slope(h):
            def loss(s):
                moved = [x + s * h * way if n == at else x for n, x in enumerate((q, k, v))]
                return (oa.forward(*moved, c.ends_host, c.scale, 1, 0.0)[0] * c.do_value).sum()
            return (loss(1) - loss(-1)) / (2 * h)

        # central differences are off by C h^2: a third of what those of twice the step differ from them
        want, wide = slope(step), slope(2 * step)
        got = (c.split(grad) * way).sum()
        off = oa.backward(q, k, v, c.split(c.out), c.lse.double().cpu().numpy(), c.do_value, c.ends_host, c.scale, 1, UNIT[0])[3 + at]
        # the forward pass's own rounding of out and lse reaches the gradient too: as much again, for each
        assert abs(got - want) <= 3 * (off * np.abs(way)).sum() + abs(wide - want) + 1e-7, (at, got, want)


@pytest.mark.parametrize("dtype", [1, 0])
def test_captured_and_on_another_stream(dtype):
    """A captured forward and backward pass, replayed over new inputs, beside eager calls on another stream."""
    c = Call(dtype, 4, 2, 64, [90, 33, 130], behind=2, seed=10)
    c.fwd(1)
    c.bwd(1)
    side = torch.cuda.Stream()
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        c.fwd(1, stream=s)
        c.bwd(1, stream=s)
    for seed in (11, 12, 13):
        e = Call(dtype, 4, 2, 64, [90, 33, 130], behind=2, seed=seed)
        for x, y in ((c.q, e.q), (c.k, e.k), (c.v, e.v), (c.do, e.do)):
            x.copy_(y)
        sync()
        graph.replay()
        with torch.cuda.stream(side):
            e.fwd(1, stream=side.cuda_stream)
            e.bwd(1, stream=side.cuda_stream)
        sync()
        for name in ("out", "lse", "dq", "dk", "dv"):
            assert torch.equal(getattr(c, name), getattr(e, name)), name


def test_offsets_past_32_bits():
    """Rows whose elements are counted past 2^31."""
    h, d, T, ld = 1, 64, 70000, 32768
    g = torch.Generator(device=DEV).manual_seed(0)
    buf = torch.empty(T, ld, dtype=torch.bfloat16, device=DEV)
    small = torch.randn(100, 4 * d, generator=g, device=DEV).bfloat16()
    buf[-100:, :4 * d] = small
    q, k, v, do = (buf[:, i * d:(i + 1) * d] for i in range(4))
    ends = torch.tensor([0, 0, T - 100, T], dtype=torch.int32, device=DEV)[[2, 3]].contiguous()
    buf[:-100, :4 * d] = 0
    out, grads = (torch.zeros(T, ld, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    lse = torch.zeros(h, T, device=DEV)
    ws = torch.empty(mi.mimose_op_packed_attention_bwd_workspace_bytes(T, h, h, d), dtype=torch.uint8, device=DEV)
    head = (ends, 2, T, h, h, d, 1, 0.125)
    mi.mimose_op_packed_attention_fwd(1, q, ld, k, ld, v, ld, out, ld, lse, *head)
    mi.mimose_op_packed_attention_bwd(1, q, ld, k, ld, v, ld, out, ld, lse, do, ld, grads, ld, grads[:, d:], ld, grads[:, 2 * d:], ld, *head,
                                      workspace=ws, workspace_bytes=ws.numel())
    sync()
    rows = lambda x: x.double().cpu().numpy().reshape(100, 1, d)  # noqa: E731
    operands = [rows(small[:, i * d:(i + 1) * d]) for i in range(4)]
    got, got_lse = rows(out[-100:, :d]), lse[:, -100:].double().cpu().numpy()
    want, want_lse, off, lse_off = oa.forward(*operands[:3], [100], 0.125, 1, UNIT[1])
    within(got, want, off, "out")
    within(got_lse, want_lse, lse_off, "lse")
    want = oa.backward(*operands[:3], got, got_lse, operands[3], [100], 0.125, 1, UNIT[1])
    for i, name in enumerate(("dq", "dk", "dv")):
        within(rows(grads[-100:, i * d:(i + 1) * d]), want[i], want[3 + i], name)


def test_nothing_to_do():
    c = Call(1, 2, 1, 64, [5], behind=4, seed=14)
    empty = torch.zeros(3, dtype=torch.int32, device=DEV)
    for n, T in ((0, c.T), (3, c.T), (1, 0)):
        c.ends, c.n_seq, c.T = empty, n, T
        c.fwd(1)
        c.bwd(1)
    sync()
    for x in (c.out, c.lse, c.dq, c.dk, c.dv):
        assert (x == KEEP).all()
