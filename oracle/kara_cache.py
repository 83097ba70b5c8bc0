"""The cache in 4 bits and eviction by accumulated weight -- TEST INFRASTRUCTURE,
NOT PRODUCT.

Plain fp64 numpy from the definitions in include/kara_q4.h and
include/kara_evict.h; only tests use it, and it shares nothing with the
library.

    q4_quantize   blocks of 32 values to codes and scale bytes
    q4_values     what they stand for
    attend        softmax attention of a sequence's last T tokens, and the weight
                  each key gets
    kept          the positions eviction keeps
"""

from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def q4_quantize(x: np.ndarray):
    """x [..., d] -> codes [..., d/2] uint8, scale bytes [..., d/32] uint8."""
    b = np.asarray(x, dtype=np.float64).reshape(x.shape[:-1] + (-1, 32))
    b = np.where(np.isnan(b), 0.0, b)
    top = np.where(np.isinf(b), 0.0, np.abs(b)).max(axis=-1)
    e = np.full(top.shape, -125, dtype=np.int64)
    nz = top > 0
    fl = np.frexp(top[nz])[1] - 1                        # floor(log2(top))
    e[nz] = fl - 2 + (top[nz] > 7.0 * np.exp2(fl - 2.0))
    e = np.clip(e, -125, 125)
    y = np.abs(b) / np.exp2(e.astype(np.float64))[..., None]
    # nearest value: the midpoints belong to the even code beside them
    code = np.zeros(y.shape, dtype=np.uint8)
    for c in range(7):
        mid = (MAGNITUDES[c] + MAGNITUDES[c + 1]) / 2
        code += (y > mid) if c % 2 == 0 else (y >= mid)
    code |= (np.signbit(b).astype(np.uint8) << 3)
    code = code.reshape(x.shape)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).astype(np.uint8)


def q4_values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """fp64 values [..., d] of codes [..., d/2] and scale bytes [..., d/32]."""
    lut = np.concatenate([MAGNITUDES, -MAGNITUDES])
    v = np.stack([lut[codes & 15], lut[codes >> 4]], axis=-1).reshape(codes.shape[:-1] + (-1,))
    return v * np.repeat(np.exp2(scales.astype(np.float64) - 127.0), 32, axis=-1)


def attend(q, k, v, scale):
    """q [T, Hq, d], k, v [n, Hkv, d] (v may be None), fp64.  Query t sits at
    position n - T + t and sees the keys up to it; one whose every logit is -inf
    gives no key a weight.  Returns out [T, Hq, d], the sums of w|v| [T, Hq, d],
    and the keys' weights [Hkv, n]."""
    T, Hq, d = q.shape
    n, Hkv = k.shape[:2]
    G = Hq // Hkv
    out, mass = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    weights = np.zeros((Hkv, n))
    for t in range(T):
        m = n - T + t + 1
        if m <= 0:
            continue
        for hq in range(Hq):
            h = hq // G
            x = scale * (k[:m, h] @ q[t, hq])
            if x.max() == -np.inf:
                continue
            w = np.exp(x - x.max())
            w /= w.sum()
            weights[h, :m] += w
            if v is not None:
                out[t, hq] = w @ v[:m, h]
                mass[t, hq] = w @ np.abs(v[:m, h])
    return out, mass, weights


def kept(weights, keep, n_sink, n_recent):
    """Positions of a row of accumulators that stay, ascending."""
    n = len(weights)
    if n <= keep:
        return np.arange(n)
    mid = np.arange(n_sink, n - n_recent)
    w = np.asarray(weights, dtype=np.float64)[mid]
    rank = np.lexsort((mid, -np.where(np.isnan(w), 0.0, w), np.isnan(w)))
    return np.sort(np.concatenate([np.arange(n_sink), mid[rank][:keep - n_sink - n_recent], np.arange(n - n_recent, n)]))
