"""Pins of the 4-bit cache's and eviction's CPU oracle: closed forms and brute force."""
import numpy as np

from oracle import kara_cache as oc


def test_codes_are_the_nearest_values():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64)) * np.exp2(rng.integers(-30, 30, (50, 1)))
    codes, scales = oc.q4_quantize(x)
    v = oc.q4_values(codes, scales)
    b, w = x.reshape(50, 2, 32), v.reshape(50, 2, 32)
    unit = np.exp2(scales.astype(float) - 127)[..., None]
    grid = np.concatenate([oc.MAGNITUDES, -oc.MAGNITUDES]) * unit[..., None]
    best = np.abs(b[..., None] - grid).min(axis=-1)
    assert np.array_equal(np.abs(b - w), best)
    top = np.abs(b).max(axis=-1, keepdims=True) / unit
    assert (top <= 7).all() and (top > 3.5).all()          # the smallest scale that keeps the top to 7 units


def test_ties_scale_borders_and_what_is_not_finite():
    def one(*values):
        x = np.zeros(32)
        x[:len(values)] = values
        c, s = oc.q4_quantize(x[None])
        return oc.q4_values(c, s)[0][:len(values)].tolist(), int(s[0, 0])

    assert one(4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.25, -2.5) == ([4, 0, 1, 1, 2, 2, 4, 0, -2], 127)
    assert one(5.0) == ([4], 127) and one(5.0001) == ([6], 127)
    assert one(7.0) == ([6], 127) and one(7.0001) == ([8], 128)
    assert one(0.0) == ([0], 2) and one(2.0 ** -140) == ([0], 2)
    assert one(2.0 ** 127 * 1.9)[1] == 252
    assert one(np.nan, 4, np.inf, -np.inf) == ([0, 4, 6, -6], 127)


def test_attention_and_weights_against_brute_force():
    rng = np.random.default_rng(2)
    T, Hq, Hkv, d, n = 5, 4, 2, 8, 3                       # two queries before the sequence's start
    q, k, v = rng.standard_normal((T, Hq, d)), rng.standard_normal((n, Hkv, d)), rng.standard_normal((n, Hkv, d))
    out, mass, w = oc.attend(q, k, v, 0.5)
    assert not out[:2].any() and (mass >= np.abs(out) - 1e-15).all()
    total = np.zeros((Hkv, n))
    for t in range(2, T):
        for hq in range(Hq):
            e = np.array([np.exp(0.5 * float(q[t, hq] @ k[i, hq // 2])) for i in range(t - 1)])
            assert np.allclose(out[t, hq], (e / e.sum()) @ v[:t - 1, hq // 2])
            total[hq // 2, :t - 1] += e / e.sum()
    assert np.allclose(w, total) and np.allclose(w.sum(), 3 * Hq)


def test_kept_positions():
    w = np.array([9, 0, 3, np.nan, 3, 1, 3, np.inf, 0, 0.5])
    assert oc.kept(w, 10, 3, 4).tolist() == list(range(10))
    assert oc.kept(w, 4, 1, 2).tolist() == [0, 7, 8, 9]
    assert oc.kept(w, 3, 0, 0).tolist() == [0, 2, 7]       # of three 3s the first
    assert oc.kept(w, 9, 0, 0).tolist() == [0, 1, 2, 4, 5, 6, 7, 8, 9]
    assert oc.kept(w, 2, 1, 1).tolist() == [0, 9]
