"""Windowed attention (include/kara_window.h) of many queries where its kernel takes other paths
than small calls do: sequences sorted by length but not split, and spans of more runs of keys
than the table in LDS holds at a time.  Against fp64 numpy."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from oracle import kara_serving as ks  # noqa: E402
from test_gpu_q8 import random_pools  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _attend(q, k, v, scale, window, sink):
    """ks.attend for finite logits, a head at a time."""
    T, Hq, d = q.shape
    n, Hkv = k.shape[:2]
    sees = ks.visible(T, n, window, sink)
    some = sees.any(1)                                     # (queries before the start: zeros)
    out, mass = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    fine = np.where(np.isfinite(v), v, 0.0)
    for hq in range(Hq):
        h = hq * Hkv // Hq
        x = np.where(sees, scale * (q[:, hq] @ k[:, h].T), -np.inf)[some]
        w = np.exp(x - x.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        out[some, hq], mass[some, hq] = w @ fine[:, h], w @ np.abs(fine[:, h])
        for pos, e in np.argwhere(~np.isfinite(v[:, h])):
            out[sees[:, pos], hq, e] += v[pos, h, e]
    return out, mass


def _check(dtype, cache, Hq, Hkv, d, bs, T, layers, lens, window, sink, odd=False):
    from paper_2607_01237_amd import kara
    print(f"\n[case] {dtype} {cache} {Hq}/{Hkv} d={d} bs={bs} T={T} layers={layers} n={len(lens)} longest={max(lens)} "
          f"window={window} sink={sink} odd={odd}", flush=True)
    rng = np.random.default_rng(len(lens) + T + bs)
    lens = np.array(lens, dtype=np.int32)
    n, longest = len(lens), int(lens.max())
    table, pages, _ = cc.table_for(rng, lens, bs, -(-longest // bs))
    p = cc.params(Hq, Hkv, d, bs, pages, table.shape[1], n, dtype)
    kw = {}
    if cache == "q8":
        host, lists = random_pools(rng, 1, pages, Hkv, bs, d)
        rows_of = lambda x, s, m: host[x][0].rows(table[s], m)  # noqa: E731
        pools = [lists[0][0], lists[1][0]]
        kw = {x + "_scales": lists[2 + i] * layers for i, x in enumerate("kv")}
    else:
        pools = [torch.from_numpy(rng.standard_normal((pages, Hkv, bs, d)).astype(np.float32)).to(cc.DT[dtype]).cuda() for _ in range(2)]
        if odd:
            # infinite values near the end, seen by the later queries alone, and far back
            for pos in (longest - 2, longest - T + 3, 40):
                pools[1][int(table[0, pos // bs]), 0, pos % bs, pos % d] = float("inf")
        host = [t.double().cpu().numpy() for t in pools]
        rows_of = lambda x, s, m: cc.rows_of(host["kv".index(x)], table, s, m, bs)  # noqa: E731
    order = rng.permutation(n).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((1, n, T, Hq, d)).astype(np.float32)).to(cc.DT[dtype])
    qs = q.cuda().expand(layers, -1, -1, -1, -1).contiguous()
    out = torch.full_like(qs, 7.0)
    need = kara.window_attention_workspace_size(p, n, layers, T, window, sink, longest)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(order), T, window, sink, qs, [pools[0]] * layers, [pools[1]] * layers, cc.gpu(table),
                          cc.gpu(lens), longest, out, ws[:need], **kw)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    for l in range(1, layers):                             # the same inputs: the same bits
        assert torch.equal(out[l].view(torch.uint8), out[0].view(torch.uint8)), l
    got, worst = out[0].double().cpu().numpy(), 0.0
    scale = 1 / np.sqrt(d)
    for j, s in enumerate(order):
        m = int(lens[s])
        q64 = q[0, j].double().numpy()
        k, v = (rows_of(x, s, m) for x in "kv")
        ref, mass = _attend(q64, k, v, scale, window, sink)
        inf = np.isinf(ref)
        assert np.array_equal(got[j][inf], ref[inf]) and np.isfinite(got[j][~inf]).all(), s
        bound = cc.attention_bound(ref, mass, cc.logit_error(q64, k, scale, 1 if dtype == "bf16" else 3), m, dtype, dtype == "bf16")
        worst = max(worst, float((np.abs(got[j][~inf] - ref[~inf]) / bound[~inf]).max()))
    print(f"[case] worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0


def _lens(n, longest, T):
    rng = np.random.default_rng(n)
    x = np.maximum(1, (rng.uniform(0, 1, n) ** 3 * longest)).astype(int)
    x[n // 2], x[n // 3] = longest, T // 2                 # (one shorter than its queries)
    return x


@pytest.mark.parametrize("dtype,cache,Hq,Hkv,d,T,n", [
    ("bf16", "rows", 16, 8, 64, 70, 70), ("bf16", "q8", 16, 8, 128, 70, 70), ("f32", "q8", 16, 8, 64, 70, 70),
    ("bf16", "rows", 8, 8, 128, 80, 64), ("bf16", "rows", 4, 1, 64, 33, 511), ("bf16", "q8", 4, 1, 64, 33, 512),
    ("bf16", "rows", 4, 1, 64, 33, 512), ("bf16", "rows", 4, 1, 64, 33, 513), ("bf16", "q8", 3, 1, 128, 300, 128)])
@pytest.mark.parametrize("window,sink", [(0, 0), (90, 5)])
def test_sequences_sorted_and_not_split(dtype, cache, Hq, Hkv, d, T, n, window, sink):
    # 512 row blocks and more, of up to 512 sequences; 511 blocks, and 513 sequences beside them
    _check(dtype, cache, Hq, Hkv, d, 16, T, 1, _lens(n, 900, T), window, sink)


@pytest.mark.parametrize("layers", [16, 64])               # keys split by their lengths, and not
@pytest.mark.parametrize("dtype,cache,d,bs,longest,window,sink,odd", [
    ("bf16", "rows", 64, 7, 9000, 0, 0, False), ("bf16", "q8", 64, 7, 9000, 0, 0, False), ("f32", "q8", 64, 7, 9000, 0, 0, False),
    ("bf16", "rows", 128, 7, 6000, 2500, 700, False), ("bf16", "q8", 128, 7, 6000, 2500, 700, False),
    ("bf16", "rows", 64, 24, 20000, 0, 0, False), ("bf16", "q8", 128, 24, 20000, 0, 0, False),
    ("bf16", "rows", 64, 16, 40000, 0, 0, False), ("bf16", "q8", 64, 16, 40000, 0, 0, False),
    ("bf16", "rows", 64, 7, 9000, 0, 0, True), ("bf16", "rows", 128, 24, 20000, 0, 0, True)])
def test_more_runs_of_keys_than_the_table_holds(dtype, cache, d, bs, longest, window, sink, odd, layers):
    # 1024 runs: of 1 key at pages of 7, 8 at 24, 16 at 16.  16 layers are 256 row blocks: the
    # long sequence's keys fall to 2 splits each, of half of them; 64 layers' are not split.
    _check(dtype, cache, 16, 8, d, bs, 70, layers, [longest, 333], window, sink, odd)
