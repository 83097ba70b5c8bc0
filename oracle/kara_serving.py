"""The cache in 8 bits, the rotating append and windowed attention -- TEST
INFRASTRUCTURE, NOT PRODUCT.

Plain fp64 numpy from the definitions in include/kara_q8.h, include/kara_rope.h
and include/kara_window.h; only tests use it, and it shares nothing with the
library.

    q8_scale      the exponent of a block
    q8_codes      e4m3 codes of values under an exponent
    q8_values     what codes under a scale byte stand for
    Q8Pool        a pool's codes and scales, appended to token by token
    turn          the rotation
    attend        windowed attention with the first tokens visible
"""

from __future__ import annotations

import numpy as np

# the magnitudes of codes 0 .. 126
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def q8_scale(block: np.ndarray) -> int:
    """The exponent e of a block of values (not finite ones are left out)."""
    mags = np.abs(block[np.isfinite(block)])
    top = mags.max() if mags.size else 0.0
    if top == 0:
        return -117
    e = int(np.frexp(top)[1]) - 1 - 8                  # floor(log2(top)) - 8
    return int(np.clip(e + (top > 448.0 * 2.0 ** e), -117, 119))


def q8_codes(x: np.ndarray, e) -> np.ndarray:
    """Codes of x under 2^e: nearest, ties to the even code; NaN 0, magnitudes past 448 to 448."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, dtype=np.float64))
    y = np.minimum(np.abs(x) / np.exp2(np.asarray(e, dtype=np.float64)), 448.0)
    up = np.minimum(np.searchsorted(E4M3, y, side="left"), 126)         # first code not below
    down = np.maximum(up - 1, 0)
    du, dd = E4M3[up] - y, y - E4M3[down]
    code = np.where((du < dd) | ((du == dd) & (up % 2 == 0)), up, down)
    code = np.where(E4M3[up] == y, up, code)
    return (code | (np.signbit(x).astype(np.int64) << 7)).astype(np.uint8)


def q8_values(codes: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """Values of codes under scale bytes that broadcast to them (a NaN code: NaN)."""
    mag = np.concatenate([E4M3, [np.nan]])[codes & 127]
    return np.where(codes >= 128, -mag, mag) * np.exp2(np.asarray(byte, dtype=np.float64) - 127.0)


class Q8Pool:
    """codes [pages][Hkv][bs][d], scales [pages][Hkv] of one layer's K or V."""

    def __init__(self, codes, scales):
        self.codes, self.scales = codes.copy(), scales.copy()

    def append(self, table_row, n, rows):
        """rows [n_new][Hkv][d] to positions n .. of the sequence with this table row, as one call."""
        bs = self.codes.shape[2]
        end = n + len(rows)
        for b in range(n // bs, -(-end // bs)):
            lo, hi = max(n, b * bs), min(end, (b + 1) * bs)
            page = table_row[b]
            for h in range(rows.shape[1]):
                new = rows[lo - n:hi - n, h]
                e = q8_scale(new)
                old = lo - b * bs
                if old > 0:
                    was = int(np.clip(int(self.scales[page, h]), 10, 246)) - 127
                    if e > was:
                        self.codes[page, h, :old] = q8_codes(q8_values(self.codes[page, h, :old], was + 127), e)
                    e = max(e, was)
                self.codes[page, h, old:old + hi - lo] = q8_codes(new, e)
                self.scales[page, h] = e + 127

    def rows(self, table_row, n):
        """Values [n][Hkv][d] of a sequence's first n positions."""
        bs = self.codes.shape[2]
        at = np.arange(n)
        pages = table_row[at // bs]
        return q8_values(self.codes[pages, :, at % bs], self.scales[pages][:, :, None])


def turn(x, pos, dim, theta=None, inv_freq=None):
    """Rows x [n][heads][d] at rotary positions pos [n]: pairs (i, i + dim/2) turned by pos * f_i."""
    half = dim // 2
    f = np.asarray(inv_freq, dtype=np.float64) if inv_freq is not None else theta ** (-2.0 * np.arange(half) / dim)
    ang = (np.asarray(pos, dtype=np.float64)[:, None] * f)[:, None]
    c, s = np.cos(ang), np.sin(ang)
    out = np.array(x, dtype=np.float64)
    a, b = out[..., :half].copy(), out[..., half:dim].copy()
    out[..., :half], out[..., half:dim] = a * c - b * s, b * c + a * s
    return out


def visible(T, n, window, sink):
    """[T][n]: whether query t, at position n - T + t, sees key k."""
    i = (n - T + np.arange(T))[:, None]
    k = np.arange(n)[None]
    return (k <= i) & ((k > i - (window or 1 << 40)) | (k < sink))


def attend(q, k, v, scale, window=0, sink=0):
    """q [T][Hq][d], k, v [n][Hkv][d], fp64: out [T][Hq][d] and the sums of w |v|.  A query
    that sees no key, or only logits of -inf, gives zeros; values that it does not see
    do not enter, those of a weight of 0 do (0 times an infinity or a NaN is NaN)."""
    T, Hq, d = q.shape
    n, Hkv = k.shape[:2]
    sees = visible(T, n, window, sink)
    out, mass = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    with np.errstate(invalid="ignore", over="ignore"):
        for hq in range(Hq):
            h = hq // (Hq // Hkv)
            for t in range(T):
                at = np.flatnonzero(sees[t])
                if not at.size:
                    continue
                x = scale * (k[at, h] @ q[t, hq])
                if np.isnan(x).any() or x.max() == np.inf:
                    out[t, hq] = np.nan
                    continue
                if x.max() == -np.inf:
                    continue
                w = np.exp(x - x.max())
                w /= w.sum()
                out[t, hq] = w @ v[at, h]
                mass[t, hq] = w @ np.abs(v[at, h])
    return out, mass
