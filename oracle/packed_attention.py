"""Attention over packed sequences with grouped heads and its gradient in 64 bits, from their definition, and how far a
computation with fp32 sums and probabilities rounded to the storage type may be from them.

Sequence s has the rows ends[s-1] .. ends[s]-1 of q [T, h, d], k, v [T, hk, d]; query head i reads head i // (h / hk) of keys.
"""
import numpy as np

F32 = 2.0 ** -24                       # half a step of fp32


def rows_of(ends):
    return [slice(a, b) for a, b in zip([0] + list(ends[:-1]), ends) if b > a]


def _scores(q, k, scale, causal):
    """Scores, minus infinity where a row does not see another, and how far fp32 sums may be off them."""
    s = scale * q @ k.T
    # d products and sums, the scale and the exponent's argument: a rounding each, of what the absolute values add up to
    off = (q.shape[1] + 4) * F32 * scale * np.abs(q) @ np.abs(k).T
    if causal:
        s = np.where(np.arange(len(q))[:, None] >= np.arange(len(k)), s, -np.inf)
    return s, off


def forward(q, k, v, ends, scale, causal, unit):
    """out, lse and the most that each may be off; unit: half a step of the storage type, relative."""
    h, hk = q.shape[1], k.shape[1]
    out, lse = np.zeros(q.shape), np.zeros((h, len(q)))
    out_off, lse_off = np.zeros(q.shape), np.zeros((h, len(q)))
    for r in rows_of(ends):
        n = r.stop - r.start
        for i in range(h):
            j = i // (h // hk)
            s, off = _scores(q[r, i], k[r, j], scale, causal)
            top = s.max(1, keepdims=True)
            e = np.exp(s - top)
            total = e.sum(1, keepdims=True)
            p = e / total
            # a probability: its score's and the maximum's error, the exponential, and what the sum is off
            worst = np.where(np.isfinite(s), off, 0.0).max(1, keepdims=True)
            rel = 2 * worst + (n + 8) * F32 + 4 * F32 * np.abs(top)
            out[r, i] = p @ v[r, j]
            lse[i, r] = (top + np.log(total))[:, 0]
            size = p @ np.abs(v[r, j])
            out_off[r, i] = (unit + rel + (n + 8) * F32) * size + unit * np.abs(out[r, i])
            lse_off[i, r] = (worst + (n + 8) * F32 + 4 * F32 * (np.abs(top) + np.abs(lse[i, r][:, None])))[:, 0]
    return out, lse, out_off, lse_off


def backward(q, k, v, out, lse, dout, ends, scale, causal, unit):
    """dq, dk, dv and the most that each may be off."""
    h, hk, d = q.shape[1], k.shape[1], q.shape[2]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    off_q, off_k, off_v = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for r in rows_of(ends):
        n = r.stop - r.start
        add = (n * (h // hk) + 8) * F32                        # sums over rows, and over the heads that share one
        for i in range(h):
            j = i // (h // hk)
            s, s_off = _scores(q[r, i], k[r, j], scale, causal)
            z = lse[i, r][:, None]
            p = np.exp(s - z)
            p_rel = s_off + 8 * F32 * (1 + np.abs(z) + np.where(np.isfinite(s), np.abs(s), 0.0))
            g, o = dout[r, i], out[r, i]
            delta = (g * o).sum(1, keepdims=True)
            dp = g @ v[r, j].T
            ds = p * (dp - delta)
            # dp and delta: sums of d products; their difference one rounding more
            ds_off = p * ((d + 4) * F32 * (np.abs(g) @ np.abs(v[r, j]).T + (np.abs(g) * np.abs(o)).sum(1, keepdims=True))) + np.abs(ds) * p_rel
            ds_all = (unit + add) * np.abs(ds) + ds_off        # rounded to the storage type as an operand, and summed
            p_all = (unit + add + p_rel) * p
            dq[r, i] += scale * ds @ k[r, j]
            dk[r, j] += scale * ds.T @ q[r, i]
            dv[r, j] += p.T @ g
            off_q[r, i] += scale * ds_all @ np.abs(k[r, j])
            off_k[r, j] += scale * ds_all.T @ np.abs(q[r, i])
            off_v[r, j] += p_all.T @ np.abs(g)
    for x, off in ((dq, off_q), (dk, off_k), (dv, off_v)):
        off += (unit + 2 * F32) * np.abs(x)                    # stored
    return dq, dk, dv, off_q, off_k, off_v
