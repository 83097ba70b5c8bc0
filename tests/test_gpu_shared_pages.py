"""Sequences that share the pages of a prefix: listed in calls of their own, one after
the other, their weights add up in the shared accumulators (include/kara_evict.h)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from oracle import kara_cache as oc  # noqa: E402
from test_gpu_evict import KINDS, Cache, _kara  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("T", [1, 20])
def test_weights_of_two_calls_add_up(kind, dtype, T):
    kara = _kara()
    rng = np.random.default_rng(T)
    lens, Hkv, G, d, bs = [300, 170, 90], 2, 4, 64, 16
    c = Cache(rng, kind, dtype, Hkv * G, Hkv, d, bs, lens)
    c.table[1, :4] = c.table[0, :4]                      # 64 tokens of one prompt
    c.table[2, :4] = c.table[0, :4]
    c.bt.copy_(torch.from_numpy(c.table))
    want, seen, delta = c.w0[0].astype(np.float64), np.zeros(c.w0.shape[1:], dtype=np.int64), 0.0
    k, v, ks, vs = c.lists("k", "v", "ks", "vs")
    for s, n in enumerate(lens):
        q = torch.from_numpy(rng.standard_normal((1, 1, T, Hkv * G, d)).astype(np.float32)).to(cc.DT[dtype])
        sq = cc.gpu(np.array([s], dtype=np.int32))
        if T == 1:
            ws = torch.empty(kara.evict_attention_workspace_size(c.p, 1, 1, 300), dtype=torch.uint8, device="cuda")
            out = torch.empty(q.shape, device="cuda")
            kara.evict_attention(c.p, sq, q.cuda(), k, v, c.weights, c.bt, c.sl, 0, 300, out, ws, k_scales=ks, v_scales=vs)
        else:
            ws = torch.empty(kara.evict_observe_workspace_size(c.p, 1, 1, T, 300), dtype=torch.uint8, device="cuda")
            kara.evict_observe(c.p, sq, T, q.cuda(), k, c.weights, c.bt, c.sl, 0, 300, ws, k_scales=ks)
        kk, q64 = c.values("k", 0, s), q[0, 0].double().numpy()
        w = oc.attend(q64, kk, None, 1 / np.sqrt(d))[2]
        delta = max(delta, cc.logit_error(q64, kk, 1 / np.sqrt(d), 3 if dtype == "bf16" else 9))
        at = np.arange(n)
        for h in range(Hkv):
            want[c.table[s][at // bs], h, at % bs] += w[h]
            seen[c.table[s][at // bs], h, at % bs] += 1
    assert (seen == 3).sum() == 64 * Hkv
    # each of three sums of T G weights off by 2 delta and its additions, and three additions to what was there
    bound = 1.05 * (want - c.w0[0]) * (2 * delta + (T * G + 16) * cc.EPS) + 2 * 3 * cc.EPS * want + 1e-30
    err = np.abs(c.w[0].double().cpu().numpy() - want) / bound
    assert float(err.max()) < 1
