"""A layer as a training program has it: one product for queries, keys and values of packed sequences, attention over them, one
product out; their gradients; and the update of both matrices with orthogonalised steps, from whose bf16 copies the next pass reads."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, sync
from oracle import muon as om
from oracle import packed_attention as oa
from test_gpu_muon import HYPER
from test_gpu_packed_attention import within

pytestmark = pytest.mark.gpu
F32, BF16 = 2.0 ** -24, 2.0 ** -8
H, HK, D, E = 6, 2, 32, 136
W = (H + 2 * HK) * D
LENGTHS = [70, 1, 0, 33, 129]
CUTS = [slice(0, H * D), slice(H * D, (H + HK) * D), slice((H + HK) * D, W)]


class Layer:
    def __init__(self, behind, seed):
        g = torch.Generator().manual_seed(seed)
        self.rows, self.T = sum(LENGTHS), sum(LENGTHS) + behind
        self.ends = torch.tensor(np.cumsum(LENGTHS), dtype=torch.int32, device=DEV)
        normal = lambda *s: torch.randn(*s, generator=g).to(DEV)  # noqa: E731
        self.x, self.dy = normal(self.T, E).bfloat16(), normal(self.T, E).bfloat16()
        self.dy[self.rows:] = 0                                   # a loss that rows of no sequence have no part in
        self.matrices = [self.matrix(normal, W, E), self.matrix(normal, E, H * D)]
        bf = lambda c: torch.zeros(self.T, c, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        self.qkv, self.dqkv, self.out, self.dout, self.y = bf(W), bf(W), bf(H * D), bf(H * D), bf(E)
        self.lse = torch.zeros(H, self.T, device=DEV)
        self.ws = torch.empty(max(16, mi.mimose_op_packed_attention_bwd_workspace_bytes(self.T, H, HK, D)), dtype=torch.uint8, device=DEV)
        self.table = mi.MuonTable(self.matrices)

    @staticmethod
    def matrix(normal, rows, cols):
        w = normal(rows, cols) / cols ** 0.5
        return dict(master=w, grad=torch.zeros_like(w), momentum=torch.zeros_like(w), lowp=w.bfloat16())

    def gemm(self, a, a_kmajor, b, b_kmajor, c, m, n, k, stream):
        mi.mimose_op_gemm(1, a, a.stride(0), a_kmajor, b, b.stride(0), b_kmajor, c, c.stride(0), int(c.dtype == torch.float32), m, n, k, stream=stream)

    def attend(self):
        return [z for x in (*(self.qkv[:, c] for c in CUTS), self.out) for z in (x, x.stride(0))]

    def run(self):
        """One training step, all of it on torch's current stream."""
        s, (first, last), T = torch.cuda.current_stream().cuda_stream, self.matrices, self.T
        shape = (self.ends, len(LENGTHS), T, H, HK, D, 1, D ** -0.5)
        self.gemm(self.x, 1, first["lowp"], 1, self.qkv, T, W, E, s)
        mi.mimose_op_packed_attention_fwd(1, *self.attend(), self.lse, *shape, stream=s)
        self.gemm(self.out, 1, last["lowp"], 1, self.y, T, E, H * D, s)
        self.gemm(self.dy, 1, last["lowp"], 0, self.dout, T, H * D, E, s)
        self.gemm(self.dy, 0, self.out, 0, last["grad"], E, H * D, T, s)
        grads = [z for x in (self.dout, *(self.dqkv[:, c] for c in CUTS)) for z in (x, x.stride(0))]
        mi.mimose_op_packed_attention_bwd(1, *self.attend(), self.lse, *grads, *shape, workspace=self.ws, workspace_bytes=self.ws.numel(), stream=s)
        self.gemm(self.dqkv, 0, self.x, 0, first["grad"], W, E, T, s)
        mi.mimose_op_muon_step(self.table, **HYPER, stream=s)

    def held(self):
        return [x for x in (self.qkv, self.out, self.lse, self.y, self.dout, self.dqkv)] + [t[k] for t in self.matrices for k in sorted(t)]


def values(x):
    return x.double().cpu().numpy()


def product(a, b, got, name):
    """got against a @ b: fp32 sums of at most that many products, and one rounding where bf16 is stored."""
    ref = a @ b
    off = (a.shape[1] + 8) * F32 * (np.abs(a) @ np.abs(b)) + (BF16 * np.abs(ref) if got.dtype == torch.bfloat16 else 0)
    within(values(got), ref, off, name)


@pytest.mark.parametrize("behind", [0, 5])
def test_steps_of_a_layer(behind):
    """Two steps, each call's results against 64 bits from what it was given."""
    layer = Layer(behind, seed=behind)
    R, heads = layer.rows, lambda x: x[:layer.rows].reshape(layer.rows, -1, D)
    for _ in range(2):
        before = [{k: values(x) for k, x in t.items()} for t in layer.matrices]
        layer.run()
        sync()
        x, dy, qkv, out, dout, dqkv = (values(t) for t in (layer.x, layer.dy, layer.qkv, layer.out, layer.dout, layer.dqkv))
        product(x, before[0]["lowp"].T, layer.qkv, "qkv")
        parts, ends = [heads(qkv[:, c]) for c in CUTS], list(np.cumsum(LENGTHS))
        ref, lse, out_off, lse_off = oa.forward(*parts, ends, D ** -0.5, 1, BF16)
        within(heads(out), ref, out_off, "out")
        got_lse = values(layer.lse)[:, :R]
        within(got_lse, lse, lse_off, "lse")
        product(out, before[1]["lowp"].T, layer.y, "y")
        product(dy, before[1]["lowp"], layer.dout, "dout")
        product(dy.T, out, layer.matrices[1]["grad"], "gradient of the last matrix")
        want = oa.backward(*parts, heads(out), got_lse, heads(dout), ends, D ** -0.5, 1, BF16)
        for c, d, off in zip(CUTS, want[:3], want[3:]):
            within(heads(dqkv[:, c]), d, off, "dqkv")
        assert (dqkv[R:] == 0).all() and (out[R:] == 0).all()     # rows of no sequence: as they were
        product(dqkv.T, x, layer.matrices[0]["grad"], "gradient of the first matrix")
        for t, b in zip(layer.matrices, before):
            w, m, off = om.step(b["master"], values(t["grad"]), b["momentum"], **HYPER)
            assert np.linalg.norm(values(t["master"]) - w) <= off
            assert torch.equal(t["lowp"], t["master"].bfloat16())


def test_captured_steps():
    """A whole step in a graph, replayed with eager work between, gives the bits of eager steps."""
    captured, eager = Layer(3, seed=7), Layer(3, seed=7)
    keep = [x.clone() for x in captured.held()]
    captured.run()                                                # before capture: what loads at a first call
    sync()
    for x, k in zip(captured.held(), keep):
        x.copy_(k)
    sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for _ in range(4):
        graph.replay()
        eager.run()
        sync()
        assert all(torch.equal(a, b) for a, b in zip(captured.held(), eager.held()))


def test_gradient_against_differences():
    """The layer's gradient of the first matrix, against differences of its loss in 64 bits along a direction."""
    layer = Layer(0, seed=11)
    layer.run()
    sync()
    x, dy, grad = values(layer.x), values(layer.dy), values(layer.matrices[0]["grad"])
    again = Layer(0, seed=11)                                     # the weights that the pass read
    first, last = (values(t["lowp"]) for t in again.matrices)
    rng = np.random.default_rng(1)
    to = rng.standard_normal(first.shape)

    def loss(w):
        parts = [(x @ w.T)[:, c].reshape(layer.rows, -1, D) for c in CUTS]
        out = oa.forward(*parts, list(np.cumsum(LENGTHS)), D ** -0.5, 1, BF16)[0]
        return (out.reshape(layer.rows, -1) @ last.T * dy).sum()

    step = 1e-5
    slope = (loss(first + step * to) - loss(first - step * to)) / (2 * step)
    # Every number that passes between calls is rounded to bf16 once (qkv, P, out, dout, dS, dqkv), each a relative error of at most
    # BF16 that is evenly spread and independent: the sum's error is at most like that of `grad` times a random vector, whose size is
    # |to's component along it| ~ |error|.  Six roundings, each of root-mean-square BF16 / sqrt(3), change the gradient by about
    # sqrt(6 / 3) BF16 times what they act on; what they act on is at most a few times the gradient.  Ten times that in all, over a
    # direction of unit entries.
    assert abs((grad * to).sum() - slope) <= 10 * 2 ** 0.5 * BF16 * np.linalg.norm(grad)
