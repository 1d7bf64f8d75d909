"""CPU oracle of the parameter update whose moments are held in 8 bits (TEST INFRASTRUCTURE ONLY).

It shares no code with the HIP library.  The update is that of oracle/optimizer.py in fp64; what is held between
two updates of a tensor are e4m3 codes of the first moment and of the square root of the second, with one scale for
each 256 elements:

    scale  = max(largest |x| of the block, 2^-100) / 448
    q      = |x| / (scale space) + u,  space = 2^(floor(log2 max(|x| / scale, 2^-6)) - 3),  u the element's dither
    code   = e4m3 of floor(q) space, with x's sign;  a root above zero whose code would be 0 gets the smallest code
    u      = floor((K element + 0x9E3779B9 update mod 2^32) / 2^12) / 2^20,  K = 0xC13FA9A9 (m), 0x91E10DA5 (root)

`step` also returns how far each q may be from the next whole number, because a sum in fp32 can land on its other side.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256
K_M, K_V, K_STEP = 0xC13FA9A9, 0x91E10DA5, 0x9E3779B9


def decode(codes):
    """Values of e4m3 codes (bias 7, no infinities, 0x7F is NaN)."""
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    e, f = (c >> 3) & 15, (c & 7).astype(np.float64)
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def dither(n, k, update):
    i = np.arange(n, dtype=np.uint64)
    return (((i * np.uint64(k) + np.uint64(update * K_STEP & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF)) >> np.uint64(12)) / 2.0 ** 20


def scales(x):
    n = len(x)
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = np.abs(np.where(np.isfinite(x), x, 0.0))
    return np.maximum(pad.reshape(-1, BLOCK).max(1), 2.0 ** -100) / 448


def encode(x, k, update, positive=False):
    """-> codes, scales, q."""
    s = scales(x)
    a = np.abs(x) / np.repeat(s, BLOCK)[:len(x)]
    with np.errstate(invalid="ignore", over="ignore"):
        space = 2.0 ** (np.floor(np.log2(np.clip(a, 2.0 ** -6, 448))) - 3)
        q = a / space + dither(len(x), k, update)
        v = np.minimum(np.floor(q) * space, 448)
    return value_code(v, x, positive), s, q


def value_code(v, x, positive):
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.floor(np.log2(np.maximum(v, 2.0 ** -6)))
        code = np.where(v < 2.0 ** -6, v * 2.0 ** 9, (e + 7) * 8 + v / 2.0 ** (e - 3) - 8)
    code = np.where(np.isfinite(x), code, 127).astype(np.int64)
    if positive:
        code = np.where((code == 0) & (x > 0), 1, code)
    return (code + 128 * (x < 0)).astype(np.uint8)


def step(p, g, m, v, m_scale, v_scale, update, lr, beta1, beta2, eps, weight_decay):
    """One update of one tensor (fp64 in, codes and scales as held); returns a dict of what is held afterwards."""
    n = len(p)
    wide = lambda s: np.repeat(np.asarray(s, dtype=np.float64), BLOCK)[:n]  # noqa: E731
    mom = beta1 * decode(m) * wide(m_scale) + (1 - beta1) * g
    var = beta2 * (decode(v) * wide(v_scale)) ** 2 + (1 - beta2) * g * g
    p = p - lr * ((mom / (1 - beta1 ** update)) / (np.sqrt(var / (1 - beta2 ** update)) + eps) + weight_decay * p)
    mc, ms, mq = encode(mom, K_M, update)
    vc, vs, vq = encode(np.sqrt(var), K_V, update, positive=True)
    return dict(p=p, m=mc, v=vc, m_scale=ms, v_scale=vs, m_q=mq, v_q=vq, moment=mom, root=np.sqrt(var))
