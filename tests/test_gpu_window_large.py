"""Windowed attention (include/kara_window.h) of more output rows than the join of split keys
takes (2^26), in calls that join nothing."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from oracle import kara_serving as ks  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("n,T,window", [(1, 16384, 16), (16384, 1, 0)], ids=["queries", "sequences"])
def test_many_output_rows(n, T, window):
    from paper_2607_01237_amd import kara
    layers, Hq, Hkv, d, bs = 64, 64, 1, 64, 16
    assert layers * n * T * Hq >= 2 ** 26
    print(f"\n[case] {layers} layers x {n} sequences x {T} queries x {Hq} heads", flush=True)
    rng = np.random.default_rng(n)
    length = T if T > 1 else 5
    lens = np.full(n, length, dtype=np.int32)
    table, pages, _ = cc.table_for(rng, lens, bs, -(-length // bs))
    p = cc.params(Hq, Hkv, d, bs, pages, table.shape[1], n, "bf16")
    k, v = (torch.randn((pages, Hkv, bs, d), device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((layers, n, T, Hq, d), device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    need = kara.window_attention_workspace_size(p, n, layers, T, window, 0, length)
    ws = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(np.arange(n, dtype=np.int32)), T, window, 0, q, [k] * layers, [v] * layers, cc.gpu(table),
                          cc.gpu(lens), length, out, ws)
    torch.cuda.synchronize()
    k64, v64 = (t.double().cpu().numpy() for t in (k, v))
    for l, s, t in [(0, 0, 0), (layers - 1, n - 1, T - 1)] + [tuple(int(x) for x in rng.integers(0, (layers, n, T))) for _ in range(20)]:
        m = length - T + t + 1
        first = max(0, m - (window or m))
        at = np.arange(first, m)
        rows = [x[table[s][at // bs], :, at % bs] for x in (k64, v64)]
        q64 = q[l, s, t:t + 1].double().cpu().numpy()
        ref, mass = ks.attend(q64, *rows, 1 / np.sqrt(d))
        bound = cc.attention_bound(ref, mass, cc.logit_error(q64, rows[0], 1 / np.sqrt(d)), len(at), "bf16", True)
        assert (np.abs(out[l, s, t].double().cpu().numpy() - ref[0]) <= bound[0]).all(), (l, s, t)
