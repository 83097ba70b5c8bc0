"""Pins of oracle/kara_serving.py: closed forms and definitions."""
import numpy as np
import pytest

from oracle import kara_serving as ks


def test_e4m3_grid():
    assert len(ks.E4M3) == 127 and ks.E4M3[0] == 0 and ks.E4M3[1] == 2.0 ** -9 and ks.E4M3[8] == 2.0 ** -6
    assert ks.E4M3[126] == 448 and ks.E4M3[0x38] == 1 and (np.diff(ks.E4M3) > 0).all()


def test_rounding_is_to_nearest_ties_to_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-500, 500, 2000), rng.uniform(-0.1, 0.1, 2000), (ks.E4M3[:-1] + ks.E4M3[1:]) / 2])
    c = ks.q8_codes(x, 0)
    back = ks.q8_values(c, 127)
    best = np.abs(np.clip(np.abs(x), 0, 448)[:, None] - ks.E4M3).min(1)
    assert np.allclose(np.abs(np.abs(back) - np.clip(np.abs(x), 0, 448)), best, rtol=0, atol=0)
    assert ((c[-126:] & 1) == 0).all()                                   # midpoints go to the even code
    torch = pytest.importorskip("torch")
    t = torch.from_numpy(np.clip(x, -448, 448)).float()
    assert np.array_equal(ks.q8_codes(t.double().numpy(), 0), t.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.0000001, 1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -117),
                                   (3.4e38, 119), (1e-44, -117)])
def test_scale(top, e):
    assert ks.q8_scale(np.array([0.0, -top, top / 3, np.nan, np.inf])) == e


def test_appending_to_a_page_keeps_the_larger_scale():
    pool = ks.Q8Pool(np.zeros((1, 1, 4, 2), np.uint8), np.zeros((1, 1), np.uint8))
    row = np.array([0])
    pool.append(row, 0, np.array([[[1.0, 0.1]]]))
    assert pool.scales[0, 0] == 127 - 8
    pool.append(row, 1, np.array([[[100.0, 0.0]]]))                    # 64 times: e = -2
    assert pool.scales[0, 0] == 127 - 2 and pool.rows(row, 2)[0, 0, 0] == 1.0
    pool.append(row, 2, np.array([[[0.5, 0.0]]]))
    assert pool.scales[0, 0] == 127 - 2 and pool.rows(row, 3)[2, 0, 0] == 0.5
    pool.append(row, 0, np.array([[[0.5, 0.0]]]))                      # the page anew
    assert pool.scales[0, 0] == 127 - 9


def test_turn():
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]])
    assert np.allclose(ks.turn(x, [0], 4, theta=100.0), x)
    y = ks.turn(x, [1], 4, theta=100.0)[0, 0]
    assert np.allclose(y[0], np.cos(1) - 3 * np.sin(1)) and np.allclose(y[2], 3 * np.cos(1) + np.sin(1))
    assert np.allclose(y[1], 2 * np.cos(0.1) - 4 * np.sin(0.1))
    assert np.allclose(ks.turn(x, [1], 2, theta=100.0)[0, 0, 2:], [3, 4])
    a, b = ks.turn(x, [7], 4, theta=100.0), ks.turn(x, [3], 4, theta=100.0)
    c, d = ks.turn(x, [107], 4, theta=100.0), ks.turn(x, [103], 4, theta=100.0)
    assert np.allclose((a * b).sum(), (c * d).sum())                    # of the distance alone


def test_attend():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((9, 2, 8)), rng.standard_normal((9, 2, 8))
    from oracle import kara_cache as oc
    full, mass = ks.attend(q, k, v, 0.3)
    ref = oc.attend(q, k, v, 0.3)
    assert np.allclose(full, ref[0]) and np.allclose(mass, ref[1])
    assert np.allclose(ks.attend(q, k, v, 0.3, window=9)[0], full)
    one = ks.attend(q, k, v, 0.3, window=1)[0]                          # itself alone
    for t in range(3):
        assert np.allclose(one[t, :2], v[6 + t, 0]) and np.allclose(one[t, 2:], v[6 + t, 1])
    v[4] = np.nan                                                      # between the first tokens and the window
    k[4] = np.inf
    got = ks.attend(q, k, v, 0.3, window=2, sink=3)[0]
    at = [0, 1, 2, 7, 8]
    assert np.allclose(got[2], oc.attend(q[2:], k[at], v[at], 0.3)[0][0])
    assert ks.visible(5, 3, 0, 0)[:2].sum() == 0                       # queries before the start
