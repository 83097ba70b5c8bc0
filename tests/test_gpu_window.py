"""Windowed attention with the first tokens visible (include/kara_window.h) against fp64
numpy, over rows and 8-bit codes, within a bound counted from its roundings."""
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


def _kara():
    from paper_2607_01237_amd import kara
    return kara


LENS = [1, 2, 700, 33, 0, 1300, 256, 257, 49]
MAX_LEN = 1299                                            # one sequence is past it


def run(dtype, cache, Hq, Hkv, d, bs, T, layers, window, sink, lens=LENS, max_len=MAX_LEN, spoil=None, unmap=True):
    """One call over random caches: outputs, and every sequence's queries, keys and values in fp64.  What no query sees is
    taken out of the table or made NaN first."""
    kara = _kara()
    rng = np.random.default_rng(Hq * 131 + d + T + window + 7 * sink)
    lens = np.array(lens, dtype=np.int32)
    max_blocks = -(-int(max(lens.max(), max_len)) // bs)
    table, pages, _ = cc.table_for(rng, lens, bs, max_blocks)
    seqs = np.concatenate([rng.permutation(len(lens)), [len(lens)]]).astype(np.int32)
    p = cc.params(Hq, Hkv, d, bs, pages, max_blocks, len(lens), dtype)
    if cache == "q8":
        host, lists = random_pools(rng, layers, pages, Hkv, bs, d)
        rows_of = lambda x, l, s, n: host[x][l].rows(table[s], n)  # noqa: E731
        pools, kw = lists[:2], dict(k_scales=lists[2], v_scales=lists[3])
    else:
        pools = [[torch.from_numpy(rng.standard_normal((pages, Hkv, bs, d)).astype(np.float32)).to(cc.DT[dtype]).cuda()
                  for _ in range(layers)] for _ in range(2)]
        if spoil:
            spoil(pools, table, lens, bs)
        host = [[t.double().cpu().numpy() for t in ts] for ts in pools]
        rows_of = lambda x, l, s, n: cc.rows_of(host["kv".index(x)][l], table, s, n, bs)  # noqa: E731
        kw = {}
    data = {}
    for s, n in enumerate(lens):
        for l in range(layers):
            data[l, s] = [rows_of(x, l, s, int(n)) for x in "kv"]
    given = table.copy()
    bad = 255 if cache == "q8" else float("nan")
    for s, n in enumerate(lens):
        if n == 0 or n > max_len:
            continue
        hidden = ~ks.visible(T, int(n), window, sink).any(0)
        for b in range(-(-int(n) // bs)):
            page = int(table[s, b])
            gone = [i for i in range(bs) if b * bs + i >= n or hidden[b * bs + i]]
            for ts in pools:
                for t in ts:
                    t[page, :, gone] = bad
            if len(gone) == bs and unmap:
                given[s, b] = (-1, pages + 7, 0)[b % 3]
    q = torch.from_numpy(rng.standard_normal((layers, len(seqs), T, Hq, d)).astype(np.float32)).to(cc.DT[dtype])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    need = kara.window_attention_workspace_size(p, len(seqs), layers, T, window, sink, max_len)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(seqs), T, window, sink, q.cuda(), *pools, cc.gpu(given), cc.gpu(lens), max_len, out,
                          ws[:need] if need else None, **kw)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    return out.double().cpu().numpy(), q.double().numpy(), data, seqs, lens


def check(case, **more):
    dtype, cache, Hq, Hkv, d, bs, T, layers, window, sink = case
    print(f"\n[case] window attention {case}", flush=True)
    max_len = more.get("max_len", MAX_LEN)
    got, q, data, seqs, lens = run(*case, **more)
    worst = 0.0
    for l in range(layers):
        for j, s in enumerate(seqs):
            n = int(lens[s]) if s < len(lens) else 0
            if n == 0 or n > max_len:
                assert not got[l, j].any(), (l, j, n)
                continue
            k, v = data[l, s]
            scale = 1 / np.sqrt(d)
            ref, mass = ks.attend(q[l, j], k, v, scale, window, sink)
            fine = np.isfinite(ref)
            assert np.array_equal(np.isnan(got[l, j]), np.isnan(ref)), (l, s)
            assert np.array_equal(got[l, j][np.isinf(ref)], ref[np.isinf(ref)]), (l, s)
            sane = np.where(np.isfinite(k), k, 0.0)
            delta = cc.logit_error(q[l, j], sane, scale, 1 if dtype == "bf16" else 3)
            bound = cc.attention_bound(ref, mass, delta, n, dtype, dtype == "bf16")
            if fine.any():
                worst = max(worst, float((np.abs(got[l, j][fine] - ref[fine]) / bound[fine]).max()))
    print(f"[case] worst error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0


CASES = [
    # dtype, cache, Hq, Hkv, d, bs, T, layers, window, sink
    ("bf16", "rows", 32, 8, 128, 16, 1, 2, 100, 4), ("bf16", "rows", 40, 8, 128, 16, 1, 1, 1, 0),
    ("bf16", "rows", 4, 4, 64, 24, 1, 1, 16, 17), ("bf16", "rows", 16, 1, 64, 16, 1, 1, 0, 0),
    ("f32", "rows", 8, 2, 128, 16, 1, 1, 300, 1), ("f32", "rows", 16, 2, 64, 7, 3, 1, 31, 200),
    ("bf16", "rows", 34, 2, 128, 16, 1, 1, 2000, 5), ("bf16", "rows", 8, 2, 128, 256, 5, 2, 64, 300),
    ("bf16", "rows", 8, 8, 64, 16, 13, 1, 5, 3), ("f32", "rows", 6, 2, 128, 16, 40, 1, 77, 9),
    ("bf16", "rows", 8, 2, 128, 16, 150, 1, 100, 4), ("bf16", "rows", 16, 8, 64, 24, 300, 1, 64, 0),
    ("bf16", "rows", 3, 1, 128, 1, 700, 1, 333, 70), ("f32", "rows", 8, 2, 64, 24, 101, 1, 500, 3),
    ("f32", "rows", 2, 2, 128, 5, 300, 1, 0, 0), ("bf16", "rows", 8, 1, 128, 16, 90, 1, 0, 7),
    ("bf16", "q8", 32, 8, 128, 16, 1, 1, 100, 4), ("bf16", "q8", 16, 2, 64, 24, 3, 1, 33, 20),
    ("f32", "q8", 8, 2, 128, 16, 2, 1, 256, 0), ("bf16", "q8", 8, 2, 128, 7, 150, 1, 100, 4),
    ("f32", "q8", 4, 2, 64, 16, 200, 1, 90, 33), ("bf16", "q8", 16, 8, 64, 256, 200, 1, 1, 1),
    ("bf16", "rows", 2, 1, 128, 16, 33, 1, 40, 2), ("bf16", "rows", 8, 1, 64, 48, 70, 2, 2**31 - 1, 2**31 - 1),
    # many heads of one KV head: a decoding step among the many rows
    ("bf16", "rows", 70, 1, 64, 16, 1, 1, 50, 4), ("bf16", "q8", 136, 1, 128, 16, 1, 1, 0, 0),
    # many units of more than 16 rows: 32 a workgroup
    ("bf16", "rows", 64, 16, 128, 16, 7, 1, 100, 4), ("bf16", "q8", 64, 16, 128, 24, 5, 1, 40, 20),
    ("bf16", "rows", 32, 16, 64, 7, 13, 1, 0, 0), ("bf16", "q8", 32, 16, 64, 16, 30, 1, 77, 3),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_attention(case):
    check(case)


@pytest.mark.parametrize("case", [
    ("bf16", "rows", 8, 2, 128, 16, 1, 1, 700, 4), ("f32", "rows", 8, 2, 64, 16, 1, 1, 700, 4),
    ("bf16", "q8", 8, 2, 128, 16, 1, 1, 0, 0), ("bf16", "rows", 4, 1, 128, 16, 200, 1, 1500, 40),
    ("bf16", "q8", 4, 1, 64, 16, 90, 1, 1500, 40), ("f32", "q8", 4, 1, 128, 16, 90, 1, 0, 40)],
    ids=lambda c: "-".join(map(str, c)))
def test_long_sequences(case):
    check(case, lens=[5000, 4097, 30], max_len=6000)


def _odd(kind):
    def spoil(pools, table, lens, bs):
        rng = np.random.default_rng(1)
        for s, n in enumerate(lens):
            for x, ts in enumerate(pools):
                for t in ts:
                    for pos in rng.choice(int(n), min(int(n), 6), replace=False) if n else []:
                        page, slot = int(table[s, pos // bs]), int(pos % bs)
                        h, e = int(rng.integers(0, t.shape[1])), int(rng.integers(0, t.shape[3]))
                        if x == 1:                            # values: of one sign, that sums are not NaN by chance
                            t[page, h, slot, e] = float("nan") if kind == "nan" else float("inf")
                        elif kind == "keys":
                            t[page, h, slot, e] = float("nan")
    return spoil


@pytest.mark.parametrize("kind", ["inf", "nan", "keys"])
@pytest.mark.parametrize("case", [
    ("bf16", "rows", 8, 2, 128, 16, 1, 1, 100, 4), ("bf16", "rows", 8, 2, 64, 16, 9, 1, 40, 4),
    ("f32", "rows", 8, 2, 128, 16, 9, 1, 40, 4), ("f32", "rows", 8, 2, 64, 24, 60, 1, 40, 4),
    ("bf16", "rows", 8, 2, 128, 16, 150, 1, 100, 4), ("bf16", "rows", 4, 2, 64, 24, 120, 1, 0, 0),
    ("bf16", "rows", 64, 16, 128, 16, 7, 1, 40, 4), ("bf16", "rows", 64, 16, 64, 16, 5, 1, 0, 0)],
    ids=lambda c: "-".join(map(str, c)))
def test_values_that_are_not_finite_reach_those_who_see_them(case, kind):
    check(case, spoil=_odd(kind))


@pytest.mark.parametrize("T", [1, 40, 200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_a_finite_logit(dtype, T):
    """Keys of -inf logits weigh nothing; a row of nothing else is zero."""
    kara = _kara()
    rng = np.random.default_rng(2)
    Hq, Hkv, d, bs, n, window = 4, 2, 64, 16, 300, 20
    table, pages, _ = cc.table_for(rng, [n], bs, 20)
    p = cc.params(Hq, Hkv, d, bs, pages, 20, 1, dtype)
    k, v = (torch.from_numpy(rng.standard_normal((pages, Hkv, bs, d)).astype(np.float32)).to(cc.DT[dtype]).cuda() for _ in range(2))
    pages_of = torch.from_numpy(table[0][np.arange(n) // bs]).long().cuda()
    slots = torch.arange(n).cuda() % bs
    for pos in range(n):
        if pos >= n - 150 or pos % 3:
            k[pages_of[pos], 0, slots[pos], 0] = float("-inf")
    q = torch.from_numpy(rng.standard_normal((1, 1, T, Hq, d)).astype(np.float32)).abs().to(cc.DT[dtype])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(1, kara.window_attention_workspace_size(p, 1, 1, T, window, 0, n)), dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(np.zeros(1, np.int32)), T, window, 0, q.cuda(), [k], [v], cc.gpu(table),
                          cc.gpu(np.array([n], np.int32)), n, out, ws)
    got = out[0, 0].double().cpu().numpy()
    k64, v64 = (t[pages_of, :, slots].double().cpu().numpy() for t in (k, v))
    ref, mass = ks.attend(q[0, 0].double().numpy(), k64, v64, 0.125, window, 0)
    dead = min(T, 150 - window + 1)                       # queries whose window holds only such keys
    assert not got[T - dead:, :2].any() and not ref[T - dead:, :2].any() and np.isfinite(got).all()
    sane = np.where(np.isfinite(k64), k64, 0.0)
    bound = cc.attention_bound(ref, mass, cc.logit_error(q[0, 0].double().numpy(), sane, 0.125, 3), n, dtype, dtype == "bf16")
    assert (np.abs(got - ref) <= bound).all()


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype,T,window", [("bf16", 1, 20), ("bf16", 8, 0), ("bf16", 200, 20), ("bf16", 200, 0), ("f32", 40, 20)])
def test_a_row_of_no_weight_is_zero_whatever_its_values(dtype, T, window, value):
    kara = _kara()
    Hq, Hkv, d, bs, n = 4, 2, 64, 16, 300
    rng = np.random.default_rng(3)
    table, pages, _ = cc.table_for(rng, [n], bs, 20)
    p = cc.params(Hq, Hkv, d, bs, pages, 20, 1, dtype)
    k, v = (torch.from_numpy(rng.standard_normal((pages, Hkv, bs, d)).astype(np.float32)).to(cc.DT[dtype]).cuda() for _ in range(2))
    k[:, 0, :, 0] = float("-inf")                         # of one head: all its rows' logits are -inf
    v[:, 0, :, ::3] = value
    q = torch.from_numpy(rng.standard_normal((1, 1, T, Hq, d)).astype(np.float32)).abs().to(cc.DT[dtype])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    ws = torch.empty(max(1, kara.window_attention_workspace_size(p, 1, 1, T, window, 0, n)), dtype=torch.uint8, device="cuda")
    kara.window_attention(p, cc.gpu(np.zeros(1, np.int32)), T, window, 0, q.cuda(), [k], [v], cc.gpu(table),
                          cc.gpu(np.array([n], np.int32)), n, out, ws)
    got = out[0, 0].float().cpu()
    assert not got[:, :2].any() and torch.isfinite(got).all() and got[:, 2:].abs().amin() > 0


def test_no_window_is_the_attention_of_all():
    """window = 0, a window past the sequence, and sinks past it: the same bits where keys are split alike."""
    kara = _kara()
    rng = np.random.default_rng(5)
    for T in (1, 100):
        lens = np.array([300, 77], dtype=np.int32)
        table, pages, _ = cc.table_for(rng, lens, 16, 19)
        p = cc.params(8, 2, 128, 16, pages, 19, 2, "bf16")
        _, lists = random_pools(rng, 1, pages, 2, 16, 128)
        q = torch.randn((1, 2, T, 8, 128), dtype=torch.bfloat16, device="cuda")
        sq = cc.gpu(np.array([1, 0], np.int32))
        outs = []
        for window, sink in ((0, 0), (300, 0), (2**31 - 1, 0), (1, 300), (5, 2**31 - 1)):
            out = torch.empty_like(q)
            ws = torch.empty(max(1, kara.window_attention_workspace_size(p, 2, 1, T, window, sink, 300)), dtype=torch.uint8, device="cuda")
            kara.window_attention(p, sq, T, window, sink, q, *lists[:2], cc.gpu(table), cc.gpu(lens), 300, out, ws,
                                  k_scales=lists[2], v_scales=lists[3])
            outs.append(out)
        out = torch.empty_like(q)
        ws = torch.empty(max(1, kara.q8_attention_workspace_size(p, 2, 1, T, 300)), dtype=torch.uint8, device="cuda")
        kara.q8_attention(p, sq, T, q, *lists, cc.gpu(table), cc.gpu(lens), 300, out, ws)
        for x in outs:
            assert torch.equal(x, out)
