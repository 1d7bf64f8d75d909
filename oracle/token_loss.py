"""CPU oracle of the losses on token log-probabilities (TEST INFRASTRUCTURE ONLY).

It shares no code with the HIP library.  Everything is fp64 numpy, written from the definitions:

    logp_t = x_t[y_t] - log sum_v exp x_t[v]                 rows whose label lies outside [0, V) are left out

    preference: s_k = sum of logp over sequence k, z_p = beta ((s_2p - r_2p) - (s_2p+1 - r_2p+1)),
                loss = mean_p (1-e) log(1 + exp(-z_p)) + e log(1 + exp(z_p))
    policy:     r = exp(logp - old), d = ref - logp, w = scale weight,
                loss = sum w (k (exp(d) - d - 1) - min(r A, clip(r, 1-lo, 1+hi) A))

The gradient of either on the logits is (d loss / d logp_t) (1[v = y_t] - softmax(x_t)[v]).  Both return, beside
the loss, `reach`: for each row a bound of the terms that d loss / d logp is made of, which tolerances are scaled by.
"""
from __future__ import annotations

import numpy as np


def scored_rows(labels, V):
    labels = np.asarray(labels)
    return (labels >= 0) & (labels < V)


def token_logprob(x, labels):
    """x[T, V] (fp64), labels[T] -> logp[T] (0 where not scored), softmax[T, V] (zeros there)."""
    T, V = x.shape
    ok = scored_rows(labels, V)
    logp, soft = np.zeros(T), np.zeros((T, V))
    for t in np.flatnonzero(ok):
        top = x[t].max()
        e = np.exp(x[t] - top)
        total = e.sum()
        soft[t] = e / total
        logp[t] = x[t, labels[t]] - top - np.log(total)
    return logp, soft


def logits_gradient(dlogp, soft, labels):
    """(d loss / d logp) (onehot - softmax) of the scored rows, zeros in the others."""
    T, V = soft.shape
    out = np.zeros((T, V))
    for t in np.flatnonzero(scored_rows(labels, V)):
        out[t] = -dlogp[t] * soft[t]
        out[t, labels[t]] += dlogp[t]
    return out


def preference_loss(x, labels, ends, ref, beta, smoothing):
    """ends: end row of each sequence.  Returns a dict with loss, logp, seq_logp, margin, dlogits, reach."""
    T, V = x.shape
    logp, soft = token_logprob(x, labels)
    ends = [int(e) for e in ends]
    P = len(ends) // 2
    seq = np.array([logp[(ends[s - 1] if s else 0):ends[s]].sum() for s in range(2 * P)])
    h = seq - np.asarray(ref, dtype=np.float64)
    z = beta * (h[0::2] - h[1::2])
    loss = np.mean((1 - smoothing) * np.logaddexp(0, -z) + smoothing * np.logaddexp(0, z))
    sig = 0.5 * (1 + np.tanh(0.5 * z))
    slope = -beta / P * ((1 - smoothing) * (1 - sig) - smoothing * sig)
    dlogp, reach = np.zeros(T), np.zeros(T)
    for s in range(2 * P):
        rows = slice(ends[s - 1] if s else 0, ends[s])
        dlogp[rows] = slope[s // 2] * (-1 if s % 2 else 1)
        reach[rows] = abs(beta) / P
    return dict(loss=loss, logp=logp, seq_logp=seq, margin=z, dlogits=logits_gradient(dlogp, soft, labels), soft=soft, reach=reach)


def policy_loss(x, labels, old, ref, advantage, weight, scale, clip_low, clip_high, kl_weight):
    """ref or weight None: no KL term, weights of 1.  Returns a dict with stats, rows, dlogits, reach."""
    T, V = x.shape
    logp, soft = token_logprob(x, labels)
    rows, dlogp, reach = np.zeros((T, 4)), np.zeros(T), np.zeros(T)
    for t in np.flatnonzero(scored_rows(labels, V)):
        w = scale * (1.0 if weight is None else float(weight[t]))
        rows[t, 0] = logp[t]
        if w == 0:
            continue
        r, A = np.exp(logp[t] - float(old[t])), float(advantage[t])
        free, held = r * A, min(max(r, 1 - clip_low), 1 + clip_high) * A
        d = 0.0 if ref is None else float(ref[t]) - logp[t]
        kl = 0.0 if ref is None else np.expm1(d) - d
        rows[t, 1:] = w * (kl_weight * kl - min(free, held)), w * kl, w * (free > held)
        dlogp[t] = w * (-kl_weight * np.expm1(d) - (free if free <= held else 0.0))
        reach[t] = abs(w) * (kl_weight * (1 + np.exp(d)) + abs(free))
    return dict(stats=rows[:, 1:].sum(0), rows=rows, dlogits=logits_gradient(dlogp, soft, labels), soft=soft, reach=reach)
