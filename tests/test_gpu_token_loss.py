"""Log-probabilities, preference loss and policy loss against the fp64 oracle, on what the device holds.

Tolerances, with u = 2^-24 the rounding of fp32.  An exponential is off by (2 |x - max| + 4) u relative (its argument
times log2 e is rounded, and the hardware's result), and |x - max| counts by the weight that exp gives it: below 32 for
every term that reaches u of the sum.  A sum over V columns has at most V / 256 + 32 roundings behind one another.  So
    lse is off by          LSE = (V / 256 + 128) u
    logp by                LSE + 4 u |logp|
and an element of the gradient, (d loss / d logp) (onehot - softmax), by reach (onehot + softmax) (LSE + slack), slack
the relative error of d loss / d logp, plus the rounding of what is stored: half a unit in the last place of bf16 (2^-8) or of fp32 (2^-24)."""
import numpy as np
import pytest
import torch

import paper_2209_02478_amd as mi
from gpu_util import DEV, TDT, quant, host, sync
from oracle import token_loss as tl

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def lse_tol(V):
    return (V / 256 + 128) * U


def workspace(T):
    return torch.empty(mi.mimose_op_token_loss_workspace_bytes(T), dtype=torch.uint8, device=DEV)


def logits_of(dtype, x, ld, offset=0, behind=7.0, unscored=None):
    """x[T, V] in a device buffer with leading dimension ld, `offset` elements behind the buffer's start; `behind`
    fills the columns from V on, NaN the rows that are not scored."""
    T, V = x.shape
    buf = torch.full((offset + T * ld + 64,), behind, dtype=TDT[dtype], device=DEV)
    rows = buf[offset:offset + T * ld].view(T, ld)
    rows[:, :V] = torch.tensor(x.astype(np.float32)).to(TDT[dtype]).to(DEV)
    if unscored is not None:
        rows[torch.tensor(unscored, device=DEV)] = float("nan")
    return rows


def inputs(seed, T, V, dtype):
    rng = np.random.default_rng(seed)
    x = quant(rng.standard_normal((T, V)) * 2.5, dtype)
    labels = rng.integers(0, V, T).astype(np.int32)
    x[np.arange(T), labels] = quant(x[np.arange(T), labels] + 6 * rng.random(T), dtype)
    labels[rng.random(T) < 0.3] = -1
    if T > 2:
        labels[T // 2] = V + 5                     # outside the vocabulary: not scored
        labels[0] = rng.integers(0, V)
    return rng, x, labels


def i32(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def f32(a):
    return torch.tensor(np.asarray(a, dtype=np.float32), device=DEV)


def check_logp(got, ref, V):
    assert np.all(np.abs(got - ref) <= np.where(ref == 0, 0, lse_tol(V) + 4 * U * np.abs(ref)))


def check_gradient(got, ref, labels, V, dtype, slack):
    """got[T, ld] against the oracle's dict; slack[T]."""
    T = len(labels)
    assert not got[:, V:].any() and not got[~tl.scored_rows(labels, V)].any()
    onehot = np.zeros((T, V))
    ok = np.flatnonzero(tl.scored_rows(labels, V))
    onehot[ok, labels[ok]] = 1
    tol = (ref["reach"] * (lse_tol(V) + slack))[:, None] * (onehot + ref["soft"]) \
        + (2.0 ** -8 if dtype == 1 else U) * np.abs(ref["dlogits"]) + 1e-37
    worst = np.abs(got[:, :V] - ref["dlogits"]) - tol
    assert worst.max() <= 0, (worst.max(), np.unravel_index(worst.argmax(), worst.shape))


# V, ld, offset in elements of the buffer: rows of 16-byte chunks and not, one column, a row longer than a block's threads hold
SHAPES = [(1, 1, 0), (1, 64, 0), (2, 8, 0), (7, 7, 1), (64, 64, 0), (1000, 1024, 0), (1003, 1003, 3), (1003, 1008, 0), (2049, 2304, 0),
          (5000, 5056, 1), (30522, 30528, 0), (50257, 50304, 0), (131000, 131072, 0), (150001, 150016, 0)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V,ld,offset", SHAPES)
def test_logprob(dtype, V, ld, offset):
    for T in (1, 5, 37):
        rng, x, labels = inputs(V + T, T, V, dtype)
        if V > 4:
            x[0, V // 3:V // 2] = -np.inf          # tokens that are ruled out
            labels[0] = V - 1
        lg = logits_of(dtype, x, ld, offset, behind=1e4, unscored=np.flatnonzero(~tl.scored_rows(labels, V)))
        ref = tl.token_logprob(x, labels)[0]
        for ws in (None, workspace(T)):
            logp = torch.full((T,), 3.0, device=DEV)
            mi.mimose_op_token_logprob(dtype, lg, ld, i32(labels), logp, T, V, ws, 0 if ws is None else ws.numel())
            sync()
            check_logp(host(logp), ref, V)


def run_preference(dtype, lg, ld, labels, ends, P, L, ref, beta, smoothing, dlogits, T, V, stream=None):
    ws = workspace(T)
    out = dict(logp=torch.full((T,), 3.0, device=DEV), seq=torch.empty(2 * P, device=DEV), margin=torch.empty(P, device=DEV),
               loss=torch.empty(1, device=DEV))
    mi.mimose_op_preference_loss(dtype, lg, ld, i32(labels), None if ends is None else i32(ends), P, L, f32(ref), beta, smoothing, dlogits,
                                 out["logp"], out["seq"], out["margin"], out["loss"], T, V, ws, ws.numel(), stream)
    sync()
    return out


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V,ld,offset", SHAPES)
@pytest.mark.parametrize("smoothing", [0.0, 0.15])
def test_preference(dtype, V, ld, offset, smoothing):
    """Pairs packed with sequences of no rows, one row and many, rows behind the last end; in place and beside; loss alone."""
    ends, T, beta = [4, 4, 5, 17, 17, 29], 31, 0.25
    rng, x, labels = inputs(V, T, V, dtype)
    labels[17:29] = -1                             # a sequence without scored rows against one without rows
    ref = rng.standard_normal(6).astype(np.float32) * 2
    want = tl.preference_loss(x, labels, ends, ref, beta, smoothing)
    bad = np.flatnonzero(~tl.scored_rows(labels, V))
    lg = logits_of(dtype, x, ld, offset, unscored=bad)
    beside = torch.full_like(torch.empty(T * ld + 8, dtype=TDT[dtype], device=DEV), 9.0)[offset % 2:offset % 2 + T * ld].view(T, ld)
    out = run_preference(dtype, lg, ld, labels, ends, 3, 0, ref, beta, smoothing, beside, T, V)
    only = run_preference(dtype, lg, ld, labels, ends, 3, 0, ref, beta, smoothing, None, T, V)
    run_preference(dtype, lg, ld, labels, ends, 3, 0, ref, beta, smoothing, lg, T, V)
    assert all(torch.equal(out[k], only[k]) for k in out)
    assert torch.equal(lg, beside)
    check_logp(host(out["logp"]), want["logp"], V)
    seq_tol = 31 * lse_tol(V) + 8 * U * np.abs(want["logp"]).sum()
    assert np.abs(host(out["seq"]) - want["seq_logp"]).max() <= seq_tol
    z_tol = 2 * beta * seq_tol + U * np.abs(want["margin"]).max()
    assert np.abs(host(out["margin"]) - want["margin"]).max() <= z_tol
    assert abs(float(out["loss"]) - want["loss"]) <= z_tol + 8 * U * want["loss"]
    check_gradient(host(beside), want, labels, V, dtype, z_tol + 16 * U)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("P,L", [(1, 1), (2, 33), (16, 3), (1, 700), (300, 2)])
def test_preference_without_ends(dtype, P, L):
    T, V, ld = 2 * P * L, 333, 336
    rng, x, labels = inputs(P + L, T, V, dtype)
    want0 = tl.token_logprob(x, labels)[0]
    ref = np.array([want0[s * L:(s + 1) * L].sum() for s in range(2 * P)]) + rng.standard_normal(2 * P)
    ref = ref.astype(np.float32)
    want = tl.preference_loss(x, labels, [(s + 1) * L for s in range(2 * P)], ref, 0.1, 0.0)
    lg = logits_of(dtype, x, ld)
    d = torch.empty_like(lg)
    out = run_preference(dtype, lg, ld, labels, None, P, L, ref, 0.1, 0.0, d, T, V)
    seq_tol = L * lse_tol(V) + 8 * U * np.abs(want["logp"]).sum()
    z_tol = 0.2 * seq_tol + U * np.abs(want["margin"]).max()
    assert np.abs(host(out["margin"]) - want["margin"]).max() <= z_tol
    assert abs(float(out["loss"]) - want["loss"]) <= z_tol + 8 * U * want["loss"]
    check_gradient(host(d), want, labels, V, dtype, z_tol + 16 * U)


def test_preference_of_no_rows_and_of_far_margins():
    """No rows at all: the loss is that of the reference alone.  Margins of +-inf and far ones stay finite where the formula does."""
    ref = np.array([100.0, -100.0, -1e4, 1e4, 0.0, 0.0], np.float32)
    out = run_preference(1, None, 64, [], [0] * 6, 3, 0, ref, 1.0, 0.0, None, 0, 64)
    assert host(out["margin"]).tolist() == [-200.0, 2e4, 0.0]
    assert abs(float(out["loss"]) - (200.0 + np.log(2)) / 3) < 1e-4
    # a chosen token that was ruled out: loss and margin are infinite, the gradient is beta / P on the chosen rows
    x = np.zeros((2, 8))
    x[0, 3] = -np.inf
    lg = logits_of(0, x, 8)
    d = torch.empty_like(lg)
    out = run_preference(0, lg, 8, [3, 1], None, 1, 1, [0.0, 0.0], 0.5, 0.0, d, 2, 8)
    assert float(out["loss"]) == np.inf and host(out["margin"])[0] == -np.inf
    assert np.allclose(host(d)[0], [0.5 / 7] * 3 + [-0.5] + [0.5 / 7] * 4, atol=1e-6)


def policy_inputs(seed, T, V, dtype):
    rng, x, labels = inputs(seed, T, V, dtype)
    logp = tl.token_logprob(x, labels)[0]
    move = rng.standard_normal(T) * 0.3
    for bound in (np.log(0.8), np.log(1.28)):      # no rounding decides which side of a bound a ratio is on
        move = np.where(np.abs(move - bound) < 1e-3, bound + 2e-3, move)
    old = (logp - move).astype(np.float32)
    ref = (logp + rng.standard_normal(T) * 0.4).astype(np.float32)
    adv = rng.standard_normal(T).astype(np.float32)
    weight = rng.random(T).astype(np.float32)
    if T > 3:
        adv[1] = 0.0
        weight[3], old[3], adv[3] = 0.0, -np.inf, np.nan     # left out of the loss whatever else it holds
    return x, labels, old, ref, adv, weight


def run_policy(dtype, lg, ld, labels, old, ref, adv, weight, scale, lo, hi, kl, dlogits, T, V, ws, stream=None):
    rows, stats = torch.full((T, 4), 3.0, device=DEV), torch.full((3,), 3.0, device=DEV)
    opt = lambda a: None if a is None else f32(a)  # noqa: E731
    mi.mimose_op_policy_loss(dtype, lg, ld, i32(labels), f32(old), opt(ref), f32(adv), opt(weight), scale, lo, hi, kl, dlogits, rows, stats,
                             T, V, ws, 0 if ws is None else ws.numel(), stream)
    sync()
    return rows, stats


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("V,ld,offset", SHAPES)
@pytest.mark.parametrize("kl", [0.0, 0.05])
def test_policy(dtype, V, ld, offset, kl):
    for T in (1, 6, 37):
        x, labels, old, ref, adv, weight = policy_inputs(V + T, T, V, dtype)
        use_ref, use_w = kl > 0 or T == 6, T != 37 or kl > 0
        if not use_w and T > 3:
            old[3], adv[3] = 0.0, 0.0
        args = (old, ref if use_ref else None, adv, weight if use_w else None, 0.125, 0.2, 0.28, kl)
        want = tl.policy_loss(x, labels, *args)
        bad = np.flatnonzero(~tl.scored_rows(labels, V))
        ws = workspace(T) if T != 6 else None
        lg = logits_of(dtype, x, ld, offset, unscored=bad)
        beside = torch.full((T, ld), 9.0, dtype=TDT[dtype], device=DEV)
        rows, stats = run_policy(dtype, lg, ld, labels, *args, beside, T, V, ws)
        rows0, stats0 = run_policy(dtype, lg, ld, labels, *args, None, T, V, ws)
        run_policy(dtype, lg, ld, labels, *args, lg, T, V, ws)
        assert torch.equal(rows, rows0) and torch.equal(stats, stats0) and torch.equal(lg, beside)
        got = host(rows)
        check_logp(got[:, 0], want["rows"][:, 0], V)
        # exp(logp - old) and exp(ref - logp) carry logp's error, relative, and their own few roundings
        slack = lse_tol(V) + 4 * U * np.abs(want["rows"][:, 0]) + 16 * U
        w = np.abs(0.125 * (weight if use_w else np.ones(T)))
        assert np.all(np.abs(got[:, 1] - want["rows"][:, 1]) <= 2 * slack * (want["reach"] + np.where(w > 0, w * np.abs(adv) * 1.28, 0)) + 1e-37)
        scale = w * (2 + np.abs(np.where(np.isfinite(ref), ref, 0) - want["rows"][:, 0]))
        assert np.all(np.abs(got[:, 2] - want["rows"][:, 2]) <= 4 * slack * scale + 1e-37)
        assert np.all(np.abs(got[:, 3] - want["rows"][:, 3]) <= 4 * U * w)
        total = np.abs(got[:, 1:]).sum(0)
        assert np.all(np.abs(host(stats) - got[:, 1:].sum(0)) <= 2 * U * total + 1e-37)
        check_gradient(host(beside), want, labels, V, dtype, 2 * slack)


def test_policy_without_rows():
    _, stats = run_policy(1, None, 64, [], [], None, [], None, 1.0, 0.2, 0.2, 0.0, None, 0, 64, None)
    assert not stats.any()


def test_policy_on_the_bounds_and_on_rows_without_an_end():
    """A ratio of exactly 1 with bounds of 0 lies on both: the gradient passes.  An upper bound of infinity holds nothing back.
    A row whose logits are all -inf has no log-probability: NaN in its own row alone."""
    x = np.zeros((3, 4))
    x[1] = -np.inf
    lg = logits_of(0, x, 4)
    old = np.full(3, np.float32(-np.log(4)))
    for adv in (2.0, -2.0):
        d = torch.empty_like(lg)
        rows, _ = run_policy(0, lg, 4, [1, 1, 2], old, None, [adv] * 3, None, 1.0, 0.0, np.inf, 0.0, d, 3, 4, None)
        got = host(d)
        assert np.isnan(got[1]).all() and np.isnan(host(rows)[1, 0])
        assert abs(got[0, 1] + adv * 0.75) < 1e-6 and abs(got[2, 2] + adv * 0.75) < 1e-6


def test_rows_beyond_32_bits_of_offset():
    """43000 rows of 50304: the last rows lie more than 2^31 elements behind the first.  Only they are scored."""
    T, V, ld = 43000, 50257, 50304
    assert T * ld > 2 ** 31
    lg = torch.full((T, ld), 3.0, dtype=torch.bfloat16, device=DEV)
    x = quant(np.random.default_rng(5).standard_normal((2, V)) * 2, 1)
    at = [42714, T - 1]
    lg[at, :V] = torch.tensor(x.astype(np.float32)).to(torch.bfloat16).to(DEV)
    labels = np.full(T, -1, np.int32)
    labels[at] = [17, V - 1]
    logp = torch.empty(T, device=DEV)
    mi.mimose_op_token_logprob(1, lg, ld, i32(labels), logp, T, V)
    sync()
    want = tl.token_logprob(x, labels[at])[0]
    check_logp(host(logp[at]), want, V)
    ref = [float(want.sum()), 0.0]
    full = tl.preference_loss(x, labels[at], [2, 2], ref, 0.1, 0.0)
    run_preference(1, lg, ld, labels, [T, T], 1, 0, ref, 0.1, 0.0, lg, T, V)
    check_gradient(host(lg[at]), full, labels[at], V, 1, 1e-4)
    assert not lg[:42714].any() and not lg[42715:T - 1].any()


def test_calls_on_another_stream_and_in_a_graph():
    """Captured once, replayed with other logits in the same memory, eager work and waits in between."""
    T, V, ld, P = 24, 1000, 1024, 2
    x, labels, old, ref, adv, weight = policy_inputs(9, T, V, 1)
    x2 = quant(x + 0.25 * np.random.default_rng(4).standard_normal(x.shape), 1)
    lg = logits_of(1, x, ld)
    lab, seq_ref = i32(labels), f32([-3.0, -2.0, -1.0, -4.0])
    o, r, a, w = f32(old), f32(ref), f32(adv), f32(weight)
    ws = workspace(T)
    ends = i32([5, 11, 12, 24])

    def outputs():
        return dict(logp=torch.zeros(T, device=DEV), seq=torch.zeros(2 * P, device=DEV), margin=torch.zeros(P, device=DEV),
                    loss=torch.zeros(1, device=DEV), d1=torch.zeros_like(lg), rows=torch.zeros(T, 4, device=DEV),
                    stats=torch.zeros(3, device=DEV), d2=torch.zeros_like(lg))

    def both(out, stream):
        mi.mimose_op_preference_loss(1, lg, ld, lab, ends, P, 0, seq_ref, 0.3, 0.1, out["d1"], out["logp"], out["seq"], out["margin"],
                                     out["loss"], T, V, ws, ws.numel(), stream)
        mi.mimose_op_policy_loss(1, lg, ld, lab, o, r, a, w, 0.5, 0.2, 0.28, 0.04, out["d2"], out["rows"], out["stats"], T, V, ws,
                                 ws.numel(), stream)

    out = outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        both(out, side.cuda_stream)
    sync()
    with torch.cuda.graph(graph, stream=side):
        both(out, side.cuda_stream)
    for values in (x, x2, x, x2):
        lg[:, :V] = torch.tensor(values.astype(np.float32)).to(torch.bfloat16).to(DEV)
        for t in out.values():
            t.fill_(5.0)
        graph.replay()
        sync()
        eager = outputs()
        both(eager, None)
        sync()
        for k in out:
            assert torch.equal(out[k], eager[k]), k


def test_directional_derivative_in_fp32():
    """The preference loss along a direction, by differences of the library's own losses: h = 1e-2 leaves h^2 / 6 of a
    third derivative that beta^3 (sum over rows)^3 bounds, and the loss's rounding over h."""
    T, V, ld = 12, 50, 52
    rng, x, labels = inputs(3, T, V, 0)
    ref, beta, h = np.float32([-2.0, -3.0]), 0.2, 1e-2
    direction = rng.standard_normal((T, V)) / np.sqrt(T)

    def loss(y, d=None):
        return float(run_preference(0, logits_of(0, y, ld), ld, labels, None, 1, 6, ref, beta, 0.0, d, T, V)["loss"])

    d = torch.empty(T, ld, device=DEV)
    lg = logits_of(0, x, ld)
    run_preference(0, lg, ld, labels, None, 1, 6, ref, beta, 0.0, d, T, V)
    slope = float((host(d)[:, :V] * direction).sum())
    found = (loss(x + h * direction) - loss(x - h * direction)) / (2 * h)
    assert abs(found - slope) <= h * h + 4 * U * T / h, (found, slope)
