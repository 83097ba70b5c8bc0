"""Eviction by accumulated attention weight (include/kara_evict.h) against fp64
numpy: outputs and accumulators within bounds counted from their roundings; kept
positions, moved rows, tables and released pages exactly."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from oracle import kara_cache as oc  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _kara():
    from paper_2607_01237_amd import kara
    return kara


class Cache:
    """A paged cache of one kind on the GPU, its host copy, and accumulators."""

    def __init__(self, rng, kind, dtype, Hq, Hkv, d, bs, lens, layers=1, max_blocks=None, scale=0.0, extra=5):
        self.kind, self.dtype, self.bs, self.d, self.layers = kind, dtype, bs, d, layers
        self.lens = np.asarray(lens, dtype=np.int32)
        self.max_blocks = max_blocks or max(1, -(-int(self.lens.max()) // bs))
        self.table, self.pages, _ = cc.table_for(rng, self.lens, bs, self.max_blocks, extra)
        self.p = cc.params(Hq, Hkv, d, bs, self.pages, self.max_blocks, len(self.lens), dtype, scale)
        shape = (layers, self.pages, Hkv, bs)
        if kind == "q4":
            self.host = {}
            for x in ("k", "v"):
                self.host[x], self.host[x + "s"] = cc.random_q4(rng, shape, d)
            self.dev = {x: cc.gpu(a) for x, a in self.host.items()}
        else:
            self.dev = {x: torch.from_numpy(rng.standard_normal(shape + (d,)).astype(np.float32)).to(cc.DT[dtype]).cuda()
                        for x in ("k", "v")}
            self.host = {x: t.float().cpu().numpy() for x, t in self.dev.items()}
        self.w0 = rng.random(shape, dtype=np.float32)
        self.w = cc.gpu(self.w0)
        self.bt, self.sl = cc.gpu(self.table), cc.gpu(self.lens)

    def lists(self, *names):
        return [list(self.dev[x].unbind(0)) if x in self.dev else None for x in names]

    @property
    def weights(self):
        return list(self.w.unbind(0))

    def values(self, which, l, s):
        """fp64 rows [n, Hkv, d]."""
        n = int(self.lens[s])
        rows = cc.rows_of(self.host[which][l], self.table, s, n, self.bs)
        if self.kind == "q4":
            return oc.q4_values(rows, cc.rows_of(self.host[which + "s"][l], self.table, s, n, self.bs))
        return rows.astype(np.float64)


def check_weights(c, seqs, n_new, max_len, per_key, T):
    """c.w against w0 plus `per_key[l][j]` ([Hkv, n] fp64, and a relative error); all
    else untouched.  A sum of T G weights in fp32, added to what was there."""
    got = c.w.double().cpu().numpy()
    seen = np.zeros(c.w0.shape, dtype=bool)
    worst, done = 0.0, set()
    G = c.p.n_q_heads // c.p.n_kv_heads
    for j, s in enumerate(seqs):
        if s < 0 or s >= len(c.lens) or s in done:
            continue
        n = int(c.lens[s])
        if n == 0 or n > max_len:
            continue
        done.add(s)
        at = np.arange(n)
        page, slot = c.table[s][at // c.bs], at % c.bs
        for l in range(c.layers):
            add, rel = per_key[l][j]
            old = np.where(at >= n - n_new, 0.0, c.w0[l, page, :, slot].T.astype(np.float64))
            want = old + add
            bound = 1.05 * add * (2 * rel + (T * G + 16) * cc.EPS) + 2 * cc.EPS * want + 1e-30
            worst = max(worst, float((np.abs(got[l, page, :, slot].T - want) / bound).max()))
            seen[l, page, :, slot] = True
    assert np.array_equal(got[~seen], c.w0[~seen].astype(np.float64))
    return worst


KINDS = [("rows", "bf16"), ("rows", "f32"), ("q4", "bf16"), ("q4", "f32")]


def count_case(kind, dtype, Hq, Hkv, d, bs, layers, n_new, lens, max_len, seqs):
    """Runs evict_attention; the worst error over its bound, of outputs and of accumulators."""
    kara = _kara()
    print(f"\n[case] count {kind} {dtype} Hq={Hq} Hkv={Hkv} d={d} bs={bs} n={len(seqs)}", flush=True)
    rng = np.random.default_rng(Hq * 7 + d + bs)
    c = Cache(rng, kind, dtype, Hq, Hkv, d, bs, lens, layers)
    seqs = np.asarray(seqs, dtype=np.int32)
    n = len(seqs)
    q = torch.from_numpy(rng.standard_normal((layers, n, Hq, d)).astype(np.float32)).to(cc.DT[dtype])
    out = torch.full(q.shape, 7.0, dtype=torch.float32, device="cuda")
    ws = torch.full((kara.evict_attention_workspace_size(c.p, n, layers, max_len),), 255, dtype=torch.uint8, device="cuda")
    k, v, ks, vs = c.lists("k", "v", "ks", "vs")
    kara.evict_attention(c.p, cc.gpu(seqs), q.cuda(), k, v, c.weights, c.bt, c.sl, n_new, max_len, out, ws, k_scales=ks,
                         v_scales=vs)
    got = out.double().cpu().numpy()
    worst, per_key = 0.0, [[None] * n for _ in range(layers)]
    terms = 1 if dtype == "bf16" else 3
    for l in range(layers):
        for j, s in enumerate(seqs):
            m = int(c.lens[s]) if 0 <= s < len(lens) else 0
            if m == 0 or m > max_len:
                assert not got[l, j].any()
                continue
            kk, vv = c.values("k", l, s), c.values("v", l, s)
            q64 = q[l, j][None].double().numpy()
            ref, mass, w = oc.attend(q64, kk, vv, 1 / np.sqrt(d))
            rel = cc.logit_error(q64, kk, 1 / np.sqrt(d), terms)
            per_key[l][j] = (w, rel)
            bound = cc.attention_bound(ref, mass, rel, m, "f32", False)
            worst = max(worst, float((np.abs(got[l, j] - ref[0]) / bound[0]).max()))
    ww = check_weights(c, seqs, n_new, max_len, per_key, 1)
    print("worst error / bound: out", worst, "weights", ww)
    return worst, ww


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,bs,layers,n_new", [(32, 8, 128, 16, 2, 1), (5, 1, 128, 24, 1, 0), (6, 6, 64, 7, 1, 3),
                                                      (32, 2, 64, 256, 1, 2000)])
def test_attention_counts(kind, dtype, Hq, Hkv, d, bs, layers, n_new):
    # the 1300-token sequence is over max_len, 5 is listed twice
    assert max(count_case(kind, dtype, Hq, Hkv, d, bs, layers, n_new, [1, 31, 0, 256, 257, 1100, 1300, 90], 1200,
                          [7, 5, 1, -1, 0, 8, 3, 4, 6, 2, 5])) < 1


@pytest.mark.parametrize("kind", ["rows", "q4"])
@pytest.mark.parametrize("layers,long,bs", [(4, 4200, 16), (2, 2500, 7), (4, 8300, 8)])
def test_attention_counts_in_large_launches(kind, layers, long, bs):
    # many units: longer splits, and more keys to a workgroup of the counting half
    lens = [long, 1, 1025, long - 1] + [40] * 60
    assert max(count_case(kind, "bf16", 8, 8, 64, bs, layers, 1, lens, long, list(range(63, -1, -1)))) < 1


def test_attention_over_rows_is_decode_attention():
    # the same splits, the same bits as the attention that does not count, where a
    # sequence has more than one split to join in order
    kara = _kara()
    rng = np.random.default_rng(8)
    c = Cache(rng, "rows", "bf16", 32, 8, 128, 16, [900, 300, 2000])
    q = torch.randn((1, 3, 32, 128), dtype=torch.bfloat16, device="cuda")
    seqs = cc.gpu(np.arange(3, dtype=np.int32))
    a, b = (torch.empty((1, 3, 32, 128), device="cuda") for _ in range(2))
    k, v = c.lists("k", "v")
    ws = torch.empty(kara.evict_attention_workspace_size(c.p, 3, 1, 2000), dtype=torch.uint8, device="cuda")
    kara.decode_attention(c.p, seqs, q, k, v, c.bt, c.sl, 2000, a, ws)
    kara.evict_attention(c.p, seqs, q, k, v, c.weights, c.bt, c.sl, 1, 2000, b, ws)
    assert float((a - b).abs().max()) <= 8 * cc.EPS * float(a.abs().max())     # (the divisions differ by a rounding)


def observe_case(kind, dtype, Hq, Hkv, d, bs, layers, T, n_new, lens, max_len, seqs):
    kara = _kara()
    print(f"\n[case] observe {kind} {dtype} Hq={Hq} Hkv={Hkv} d={d} bs={bs} T={T}", flush=True)
    rng = np.random.default_rng(Hq + d * 3 + T)
    c = Cache(rng, kind, dtype, Hq, Hkv, d, bs, lens, layers)
    seqs = np.asarray(seqs, dtype=np.int32)
    n = len(seqs)
    q = torch.from_numpy(rng.standard_normal((layers, n, T, Hq, d)).astype(np.float32)).to(cc.DT[dtype])
    ws = torch.full((kara.evict_observe_workspace_size(c.p, n, layers, T, max_len),), 255, dtype=torch.uint8, device="cuda")
    k, ks = c.lists("k", "ks")
    kara.evict_observe(c.p, cc.gpu(seqs), T, q.cuda(), k, c.weights, c.bt, c.sl, n_new, max_len, ws, k_scales=ks)
    terms = 1 if dtype == "bf16" else 3
    per_key = [[None] * n for _ in range(layers)]
    for l in range(layers):
        for j, s in enumerate(seqs):
            if not 0 <= s < len(lens) or lens[s] == 0:
                continue
            kk, q64 = c.values("k", l, s), q[l, j].double().numpy()
            per_key[l][j] = (oc.attend(q64, kk, None, 1 / np.sqrt(d))[2], cc.logit_error(q64, kk, 1 / np.sqrt(d), 3 * terms))
    worst = check_weights(c, seqs, n_new, max_len, per_key, T)
    print("worst error / bound", worst)
    return worst


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,bs,layers,T,n_new", [
    (32, 8, 128, 16, 1, 1, 1), (8, 2, 128, 24, 2, 33, 33), (6, 2, 64, 7, 1, 200, 0), (16, 1, 64, 256, 1, 70, 5),
    (40, 2, 128, 16, 1, 13, 2000)])
def test_observe(kind, dtype, Hq, Hkv, d, bs, layers, T, n_new):
    assert observe_case(kind, dtype, Hq, Hkv, d, bs, layers, T, n_new, [1, 63, 0, 64, 65, 700, 900, 129], 800,
                        [7, 5, 1, -1, 0, 8, 3, 4, 6, 2, 5]) < 1


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hq,Hkv,d,bs,T,n_new,lens,seqs", [
    (10, 2, 128, 16, 300, 300, [2600, 299, 1700], [0, 2, 1]),       # keys split, rows in parts, more queries than tokens
    (4, 4, 64, 24, 600, 0, [601, 4100], [1, 0, 1]),                 # a sequence twice, its parts added once
    (3, 1, 64, 16, 5, 1, [9000], [0]),                              # the most splits of few rows
    (8, 2, 128, 24, 33, 40, [1500, 30, 1, 32, 1100], [3, 0, 2, 4, 1]),   # few rows in several workgroups, some without keys
    (4, 4, 64, 7, 7, 7, [2100, 6, 129], [2, 0, 1])])
def test_observe_in_pieces(kind, dtype, Hq, Hkv, d, bs, T, n_new, lens, seqs):
    assert observe_case(kind, dtype, Hq, Hkv, d, bs, 1, T, n_new, lens, max(lens), seqs) < 1


def test_observe_large_logits():
    # logits of some hundreds: exponentials that overflow without the maximum, and rows past the last
    kara = _kara()
    rng = np.random.default_rng(21)
    c = Cache(rng, "rows", "bf16", 3, 1, 64, 16, [300], scale=4.0)
    q = torch.from_numpy(rng.standard_normal((1, 1, 7, 3, 64)).astype(np.float32)).bfloat16()
    ws = torch.empty(kara.evict_observe_workspace_size(c.p, 1, 1, 7, 300), dtype=torch.uint8, device="cuda")
    kara.evict_observe(c.p, cc.gpu(np.zeros(1, dtype=np.int32)), 7, q.cuda(), c.lists("k")[0], c.weights, c.bt, c.sl, 300, 300, ws)
    kk, q64 = c.values("k", 0, 0), q[0, 0].double().numpy()
    w = oc.attend(q64, kk, None, 4.0)[2]
    assert check_weights(c, [0], 300, 300, [[(w, cc.logit_error(q64, kk, 4.0))]], 7) < 1


def run_evict(c, seqs, keep, n_sink, n_recent, max_len, commit=True, given=True):
    kara = _kara()
    n, L, H = len(seqs), c.layers, c.p.n_kv_heads
    kept = torch.full((L, n, H, keep), 99, dtype=torch.int32, device="cuda")
    freed = torch.full((n, c.max_blocks), 99, dtype=torch.int32, device="cuda")
    n_freed, status = (torch.full((n,), 99, dtype=torch.int32, device="cuda") for _ in range(2))
    k, v, ks, vs = c.lists("k", "v", "ks", "vs")
    ws = torch.full((4 * n if given else kara.evict_workspace_size(c.p, n, L, keep),), 255, dtype=torch.uint8, device="cuda")
    kara.evict_tokens(c.p, cc.gpu(np.asarray(seqs, dtype=np.int32)), keep, n_sink, n_recent, k, v, c.weights, c.bt, c.sl,
                      max_len, commit, status, ws, kept=kept if given else None, freed=freed if commit else None,
                      n_freed=n_freed if commit else None, k_scales=ks, v_scales=vs)
    torch.cuda.synchronize()
    return kept.cpu().numpy(), freed.cpu().numpy(), n_freed.cpu().numpy(), status.cpu().numpy()


def check_evict(c, seqs, flagged, keep, n_sink, n_recent, res, commit=True, given=True):
    """The whole state after a cut; `flagged`: {listing: status}."""
    kept, freed, n_freed, status = res
    host = {x: (t.float() if t.dtype == torch.bfloat16 else t).cpu().numpy() for x, t in c.dev.items()}
    want = {x: a.copy() for x, a in c.host.items()}
    w_want, table, lens = c.w0.copy(), c.table.copy(), c.lens.copy()
    for j, s in enumerate(seqs):
        assert status[j] == flagged.get(j, 0), (j, status[j])
        n = 0 if j in flagged else int(c.lens[s])
        new = min(n, keep)
        ob, nb = -(-n // c.bs), -(-new // c.bs)
        if commit:
            assert n_freed[j] == ob - nb
            row = c.table[s] if j not in flagged else None
            assert freed[j].tolist() == ([] if j in flagged else row[nb:ob].tolist()) + [-1] * (c.max_blocks - (ob - nb))
        for l in range(c.layers):
            for h in range(c.p.n_kv_heads):
                at = np.arange(n)
                if n:
                    page, slot = c.table[s][at // c.bs], at % c.bs
                    pos = oc.kept(c.w0[l, page, h, slot], keep, n_sink, n_recent)
                else:
                    pos = at
                if given:
                    assert kept[l, j, h].tolist() == pos.tolist() + [-1] * (keep - len(pos)), (l, j, h)
                if n > keep:
                    for x in want:
                        want[x][l, page[:keep], h, slot[:keep]] = c.host[x][l, page[pos], h, slot[pos]]
                    w_want[l, page[:keep], h, slot[:keep]] = c.w0[l, page[pos], h, slot[pos]]
        if commit and j not in flagged:
            table[s, nb:ob] = -1
            lens[s] = new
    for x in want:
        assert np.array_equal(host[x], want[x]), x
    assert np.array_equal(c.w.cpu().numpy().view(np.int32), w_want.view(np.int32))
    assert np.array_equal(c.bt.cpu().numpy(), table) and np.array_equal(c.sl.cpu().numpy(), lens)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hkv,d,bs,layers,keep,n_sink,n_recent", [
    (8, 128, 16, 2, 200, 4, 50), (1, 64, 7, 3, 33, 0, 0), (3, 128, 256, 1, 300, 0, 300), (2, 64, 24, 1, 1, 0, 0),
    (2, 128, 16, 1, 299, 299, 0), (2, 64, 16, 1, 40, 30, 10)])
def test_evict(kind, dtype, Hkv, d, bs, layers, keep, n_sink, n_recent):
    print(f"\n[case] evict {kind} {dtype} Hkv={Hkv} d={d} bs={bs} keep={keep}", flush=True)
    rng = np.random.default_rng(keep + d + bs)
    c = Cache(rng, kind, dtype, Hkv, Hkv, d, bs, [500, keep, keep + 1, 0, 1, 700, 257, 333], layers)
    seqs = [5, 0, 3, 2, 1, 4, 6]                      # 7 is idle
    check_evict(c, seqs, {}, keep, n_sink, n_recent, run_evict(c, seqs, keep, n_sink, n_recent, 700))


def special(rng, w):
    """Accumulators that try the ranking: ties, zeros of both signs, NaN, infinities, negative, subnormal."""
    u = rng.random(w.shape)
    for lo, v in ((0.0, 0.0), (0.2, -0.0), (0.3, 0.5), (0.6, np.nan), (0.65, np.inf), (0.66, -np.inf), (0.67, -1.5),
                  (0.7, 1e-42), (0.75, 0.5000001)):
        w[u >= lo] = v
    w[u >= 0.8] = rng.random(int((u >= 0.8).sum())).astype(np.float32)


@pytest.mark.parametrize("keep", [1, 60, 140, 250, 390])
def test_evict_ranks_awkward_weights(keep):
    rng = np.random.default_rng(keep)
    c = Cache(rng, "q4", "bf16", 4, 4, 64, 16, [400, 397, 300])
    special(rng, c.w0)
    c.w.copy_(torch.from_numpy(c.w0))
    sink, recent = min(2, keep - 1), min(5, keep // 2)
    check_evict(c, [0, 1, 2], {}, keep, sink, recent, run_evict(c, [0, 1, 2], keep, sink, recent, 400))


@pytest.mark.parametrize("given,commit", [(False, True), (True, False)])
def test_evict_without_outputs(given, commit):
    rng = np.random.default_rng(17)
    c = Cache(rng, "rows", "bf16", 2, 2, 128, 16, [500, 100])
    check_evict(c, [1, 0], {}, 90, 4, 20, run_evict(c, [1, 0], 90, 4, 20, 500, commit, given), commit, given)


def test_evict_long_rows():
    # more candidates than fit in LDS, tables and kept sets that do not either; all weights equal in one
    rng = np.random.default_rng(18)
    c = Cache(rng, "q4", "bf16", 1, 1, 64, 16, [40000, 20000, 16390])
    at = np.arange(20000)
    c.w0[0, c.table[1][at // 16], 0, at % 16] = 0.25
    c.w.copy_(torch.from_numpy(c.w0))
    check_evict(c, [0, 1, 2], {}, 15000, 4, 1000, run_evict(c, [0, 1, 2], 15000, 4, 1000, 40000))


def test_evict_leaves_flagged_sequences():
    kara = _kara()
    rng = np.random.default_rng(19)
    c = Cache(rng, "rows", "f32", 2, 2, 64, 16, [200] * 9, max_blocks=16)
    c.table[1, 12] = c.pages
    c.table[2, 0] = -1
    c.table[3, 5] = c.table[3, 9]
    c.lens[4], c.lens[5] = 230, -3
    c.bt.copy_(torch.from_numpy(c.table))
    c.sl.copy_(torch.from_numpy(c.lens))
    seqs = [0, 1, 2, 3, 4, 5, 6, 6, -1, 9, 8]
    dup, win = kara.SEQ_DUP_TRIGGER, kara.SEQ_BAD_WINDOW
    flagged = {1: kara.SEQ_BAD_PAGE, 2: kara.SEQ_BAD_PAGE, 3: kara.SEQ_DUP_PAGE, 4: win, 5: win, 6: dup, 7: dup,
               8: kara.SEQ_BAD_INDEX, 9: kara.SEQ_BAD_INDEX}
    check_evict(c, seqs, flagged, 100, 4, 20, run_evict(c, seqs, 100, 4, 20, 220))


def test_evict_from_a_pool_of_many_pages():
    # more pages than the check of doubled ones keeps bits for
    kara = _kara()
    rng = np.random.default_rng(23)
    c = Cache(rng, "q4", "bf16", 1, 1, 64, 1, [300, 9000, 200, 250], extra=270000)
    c.table[2, 7] = c.table[2, 150]
    c.table[3, 249] = c.pages
    c.bt.copy_(torch.from_numpy(c.table))
    flagged = {2: kara.SEQ_DUP_PAGE, 0: kara.SEQ_BAD_PAGE}
    check_evict(c, [3, 0, 2, 1], flagged, 120, 4, 20, run_evict(c, [3, 0, 2, 1], 120, 4, 20, 9000))


def test_far_rows():
    # rows past 4 GiB of a pool: counted, observed and cut
    kara = _kara()
    rng = np.random.default_rng(31)
    d, Hkv, bs, n, keep = 128, 8, 256, 700, 300
    pages = (1 << 32) // (2 * d * Hkv * bs) + 40
    p = cc.params(16, Hkv, d, bs, pages, 3, 1, "bf16")
    pool = [torch.empty((pages, Hkv, bs, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    w = torch.zeros((pages, Hkv, bs), device="cuda")
    table = np.array([[pages - 1, pages - 30, pages - 7]], dtype=np.int32)
    at = np.arange(n)
    page, slot = table[0][at // bs], at % bs
    where = torch.from_numpy(table[0]).long().cuda()
    rows = [torch.from_numpy(rng.standard_normal((3, Hkv, bs, d)).astype(np.float32)).bfloat16() for _ in range(2)]
    for t, r in zip(pool, rows):
        t[where] = r.cuda()
    kk, vv = (r.double().numpy()[at // bs, :, slot] for r in rows)
    bt, sl, sq = cc.gpu(table), cc.gpu(np.array([n], dtype=np.int32)), cc.gpu(np.zeros(1, dtype=np.int32))
    size = max(kara.evict_attention_workspace_size(p, 1, 1, n), kara.evict_observe_workspace_size(p, 1, 1, 50, n),
               kara.evict_workspace_size(p, 1, 1, keep))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    q = torch.from_numpy(rng.standard_normal((1, 1, 50, 16, d)).astype(np.float32)).bfloat16()
    kara.evict_observe(p, sq, 50, q.cuda(), [pool[0]], [w], bt, sl, n, n, ws)
    out = torch.empty((1, 1, 16, d), device="cuda")
    kara.evict_attention(p, sq, q[:, :, 0].contiguous().cuda(), [pool[0]], [pool[1]], [w], bt, sl, 0, n, out, ws)
    q64 = q[0, 0].double().numpy()
    delta = cc.logit_error(q64, kk, 1 / np.sqrt(d), 3)
    ref, mass, one = oc.attend(q64[:1], kk, vv, 1 / np.sqrt(d))
    assert (np.abs(out[0, 0].double().cpu().numpy() - ref[0]) <= cc.attention_bound(ref, mass, delta, n, "f32", False)[0]).all()
    want = oc.attend(q64, kk, None, 1 / np.sqrt(d))[2] + one
    got = w[where].cpu().numpy()[at // bs, :, slot].T
    assert (np.abs(got - want) <= 1.05 * want * (2 * delta + (51 * 2 + 16) * cc.EPS) + 2 * cc.EPS * want).all()
    kept = torch.empty((1, 1, Hkv, keep), dtype=torch.int32, device="cuda")
    status = torch.empty(1, dtype=torch.int32, device="cuda")
    kara.evict_tokens(p, sq, keep, 4, 50, [pool[0]], [pool[1]], [w], bt, sl, n, False, status, ws, kept=kept)
    assert status.item() == 0
    to = np.arange(keep)
    for t, r in zip((*pool, w), (*rows, None)):
        a = t[where].float().cpu().numpy()[to // bs, :, to % bs]
        for h in range(Hkv):
            pos = oc.kept(got[h], keep, 4, 50)
            assert kept[0, 0, h].tolist() == pos.tolist()
            assert np.array_equal(a[:, h], got[h][pos] if r is None else r.float().numpy()[pos // bs, h, pos % bs])
