"""The rotating append's sines and cosines (include/kara_rope.h) where they are small: an angle
that lies next to a multiple of a quarter turn, to the last bits of fp32."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# Pairs (1, 0) turn to (cos, sin).  In half turns an angle is a + b, a rounded to fp32 and b
# what the rounding left, at most half a step of a: sin = sin a + b cos a.  sin a and cos a are
# off by 4 units in the last place (2^-21 of them).  Where sin a is not 0, a is a whole number of
# steps from where it is, so that b cos a is at most half of it and the sum at least half: its
# error is under 3 * 2^-21 of it.  Where it is 0 the result is b cos a, as near.  Its roundings to
# fp32: 2 * 2^-24.  Together 2^-19 of the result.  The angle itself, position * f / 2 pi turns
# formed and reduced in 64 bits: 4 roundings of 2^-53 of at most `turns` turns, times 2 pi.
def test_next_to_quarter_turns():
    from paper_2607_01237_amd import kara
    Hq, Hkv, d, bs, n_new = 2, 1, 128, 16, 3
    half = d // 2
    quarter = np.arange(half) % 16 + 1                     # f: a few steps of fp32 around quarter turns
    f = np.float32(quarter * (np.pi / 2))
    for i in range(half):
        for _ in range(i // 16):
            f[i] = np.nextafter(f[i], np.float32(1e9 if i % 2 else 0))
    table, p = np.arange(1, dtype=np.int32)[None], cc.params(Hq, Hkv, d, bs, 1, 1, 1, "f32")
    x = np.zeros((1, 1, n_new, 1, d), dtype=np.float32)
    x[..., :half] = 1.0
    k = torch.from_numpy(x).cuda()
    q = k.expand(1, 1, n_new, Hq, d).contiguous()
    pools = [[torch.zeros((1, Hkv, bs, d), device="cuda")] for _ in range(2)]
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    q_out = torch.empty_like(q)
    kara.rope_append(p, kara.make_rope(dim=d, inv_freq=cc.gpu(f)), cc.gpu(np.zeros(1, np.int32)), k, k, *pools, cc.gpu(table),
                     cc.gpu(np.zeros(1, np.int32)), status, rope_pos=cc.gpu(np.ones(1, np.int32)), q=q, q_out=q_out)
    assert status.tolist() == [0]
    angle = (1 + np.arange(n_new))[:, None] * f.astype(np.float64)         # exact
    ref = np.concatenate([np.cos(angle), np.sin(angle)], axis=-1)
    assert (np.abs(ref) < 1e-5).sum() > half                # the small ones are there
    turns = angle.max() / (2 * np.pi)
    bound = 2.0 ** -19 * np.abs(ref) + 4 * 2.0 ** -53 * turns * 2 * np.pi
    for name, got in (("k", pools[0][0][0, 0, :n_new]), ("q, head 0", q_out[0, 0, :, 0]), ("q, head 1", q_out[0, 0, :, 1])):
        worst = float((np.abs(got.double().cpu().numpy() - ref) / bound).max())
        print(f"[case] {name}: worst error / bound {worst:.3f}", flush=True)
        assert worst <= 1.0, name
