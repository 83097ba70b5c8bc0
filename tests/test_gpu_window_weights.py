"""How many bits windowed attention (include/kara_window.h) holds its weights in: two keys
whose values cancel, 1 and -1, leave the difference of their weights as the result."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# Logits 0 and -x give weights 1 and p = exp(-x), and the result (1 - p) / (1 + p).  p is off
# by the exponential's own error, 2 units in the last place of fp32 below 1 (2^-23: the
# argument's is of x's size, and far less), and by what it is held in, below 1:
#   24 bits (three bf16 terms, or fp32 itself)       nothing
#   16 bits (two terms: the first 8 bits cut off, at most 2^-8 left, rounded to 8)   2^-17
#   bf16                                             2^-9
# The result moves by 2 / (1 + p)^2 of that.  The sum of products passes values of size 1: two
# roundings there (2^-23).  Then the division and the result's own rounding.
HELD = {24: 0.0, 16: 2.0 ** -17, 8: 2.0 ** -9}

CASES = [
    # dtype, cache, query heads of one KV head, d, bits of a weight, x from 2^-e to 2^(1-e)
    ("bf16", "rows", 8, 64, 24, 12), ("bf16", "rows", 16, 128, 24, 12), ("bf16", "rows", 24, 64, 24, 12),
    ("bf16", "rows", 24, 128, 24, 12), ("bf16", "rows", 64, 128, 24, 12), ("bf16", "q8", 8, 64, 16, 7), ("bf16", "q8", 24, 128, 16, 7),
    ("bf16", "q8", 64, 64, 16, 7), ("bf16", "rows", 65, 128, 8, 2), ("bf16", "q8", 136, 64, 8, 2),
    ("f32", "rows", 8, 64, 24, 12), ("f32", "rows", 80, 128, 24, 12), ("f32", "q8", 8, 128, 24, 12), ("f32", "q8", 72, 64, 24, 12),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_a_small_difference_of_weights(case):
    from paper_2607_01237_amd import kara
    dtype, cache, G, d, bits, e = case
    print(f"\n[case] weights {case}", flush=True)
    n, bs = 256, 16                                        # sequences of two tokens, a page each
    steps = 8 if cache == "q8" else 128
    m = steps + np.arange(n) % steps                       # x = m / steps 2^-e, exact in codes as in bf16
    x = m / steps * 2.0 ** -e
    at = np.arange(n) % d                                  # the element that makes the logit
    k, v = np.zeros((n, 1, bs, d)), np.ones((n, 1, bs, d))
    k[np.arange(n), 0, 1, at] = -x
    v[:, :, 1] = -1.0
    kw = {}
    if cache == "q8":
        codes = np.zeros(k.shape, dtype=np.uint8)
        codes[np.arange(n), 0, 1, at] = 0xb8 | (m - 8)     # -m / 8 of the scale's units
        k_pool, v_pool = cc.gpu(codes), cc.gpu(np.where(v > 0, 0x38, 0xb8).astype(np.uint8))
        kw = dict(k_scales=[torch.full((n, 1), 127 - e, dtype=torch.uint8, device="cuda")],
                  v_scales=[torch.full((n, 1), 127, dtype=torch.uint8, device="cuda")])
    else:
        k_pool, v_pool = (torch.from_numpy(t).to(cc.DT[dtype]).cuda() for t in (k, v))
        assert np.array_equal(k_pool.double().cpu().numpy(), k)
    p = cc.params(G, 1, d, bs, n, 1, n, dtype, scale=1.0)
    q = torch.zeros((1, n, 1, G, d), dtype=cc.DT[dtype])
    q[0, torch.arange(n), 0, :, torch.from_numpy(at)] = 1.0
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(1, kara.window_attention_workspace_size(p, n, 1, 1, 0, 0, 2)), dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(np.arange(n, dtype=np.int32)), 1, 0, 0, q.cuda(), [k_pool], [v_pool],
                          cc.gpu(np.arange(n, dtype=np.int32)[:, None]), cc.gpu(np.full(n, 2, np.int32)), 2, out, ws, **kw)
    got = out[0, :, 0].double().cpu().numpy()
    w = np.exp(-x)
    ref = ((1 - w) / (1 + w))[:, None, None]
    moved = ((2.0 ** -23 + HELD[bits]) * 2 / (1 + w - HELD[bits]) ** 2 + 2.0 ** -23 / (1 + w))[:, None, None]
    bound = moved + (2.0 ** -8 if dtype == "bf16" else 0.0) * (ref + moved) + 2.0 ** -22 * ref
    worst = float((np.abs(got - ref) / bound).max())
    print(f"[case] worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0
