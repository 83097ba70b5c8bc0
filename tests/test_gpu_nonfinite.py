"""Infinities in keys and queries, and NaN where no sequence reaches, through the
attentions of include/kara_q4.h and include/kara_evict.h, against fp64 numpy."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from oracle import kara_cache as oc  # noqa: E402
from test_gpu_evict import KINDS, Cache, check_weights  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _kara():
    from paper_2607_01237_amd import kara
    return kara


def spoil_the_rest(c):
    """NaN (scales of infinity) in every slot that no sequence reaches."""
    free = np.ones((c.pages, c.bs), dtype=bool)
    for s, n in enumerate(c.lens):
        at = np.arange(n)
        free[c.table[s][at // c.bs], at % c.bs] = False
    at = torch.from_numpy(free).cuda()[None, :, None, :]
    for x in ("ks", "vs") if c.kind == "q4" else ("k", "v"):
        c.dev[x].masked_fill_(at[..., None], 255 if c.kind == "q4" else float("nan"))


def put_key(c, s, pos, e, value):
    """Element e of a position's key in every layer and head (rows)."""
    page, slot = c.table[s][pos // c.bs], pos % c.bs
    c.host["k"][:, page, :, slot, e] = value
    c.dev["k"][:, page, :, slot, e] = value


def queries(rng, c, n, T):
    q = rng.standard_normal((c.layers, n, T, c.p.n_q_heads, c.d)).astype(np.float32)
    return torch.from_numpy(q).to(cc.DT[c.dtype])


def run(c, fn, seqs, q, T, n_new, max_len):
    """The operator's output [layers][n][T][Hq][d], None from the one that has none."""
    kara = _kara()
    n, L = len(seqs), c.layers
    sq = cc.gpu(np.asarray(seqs, dtype=np.int32))
    k, v, ks, vs = c.lists("k", "v", "ks", "vs")
    out = torch.full(q.shape, 7.0, dtype=torch.float32 if fn == "count" else q.dtype, device="cuda")
    size = {"count": lambda: kara.evict_attention_workspace_size(c.p, n, L, max_len),
            "observe": lambda: kara.evict_observe_workspace_size(c.p, n, L, T, max_len),
            "q4": lambda: kara.q4_attention_workspace_size(c.p, n, L, T, max_len)}[fn]()
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    if fn == "count":
        kara.evict_attention(c.p, sq, q.cuda(), k, v, c.weights, c.bt, c.sl, n_new, max_len, out, ws, k_scales=ks, v_scales=vs)
    elif fn == "observe":
        kara.evict_observe(c.p, sq, T, q.cuda(), k, c.weights, c.bt, c.sl, n_new, max_len, ws, k_scales=ks)
        return None
    else:
        kara.q4_attention(c.p, sq, T, q.cuda(), k, v, ks, vs, c.bt, c.sl, max_len, out, ws)
    return out.double().cpu().numpy()


def check(c, fn, seqs, q, T, n_new, max_len):
    """The operator against the definition: infinities enter it as they are, and count as 0 in the error bounds."""
    got = run(c, fn, seqs, q, T, n_new, max_len)
    terms = (1 if c.dtype == "bf16" else 3) * (3 if fn == "observe" else 1)
    scale = 1 / np.sqrt(c.d)
    worst, per_key = 0.0, [[None] * len(seqs) for _ in range(c.layers)]
    for l in range(c.layers):
        for j, s in enumerate(seqs):
            kk, vv, q64 = c.values("k", l, s), c.values("v", l, s), q[l, j].double().numpy()
            ref, mass, w = oc.attend(q64, kk, vv, scale)
            finite = [np.where(np.isfinite(x), x, 0.0) for x in (q64, kk)]
            delta = cc.logit_error(*finite, scale, terms)
            per_key[l][j] = (w, delta)
            if got is not None:
                own = c.dtype if fn == "q4" else "f32"
                bound = cc.attention_bound(ref, mass, delta, len(kk), own, own == "bf16")
                worst = max(worst, float(np.nan_to_num(np.abs(got[l, j] - ref) / bound, nan=np.inf).max()))
    if fn != "q4":
        assert np.isfinite(c.w.cpu().numpy()).all()
        worst = max(worst, check_weights(c, seqs, n_new, max_len, per_key, T))
    print("worst error / bound", worst)
    return worst


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fn,Hq,Hkv,d,bs,T,lens", [
    ("count", 8, 2, 128, 16, 1, [300, 1500, 40]), ("count", 6, 6, 64, 7, 1, [257, 2100, 33]),
    ("observe", 8, 2, 128, 16, 40, [300, 1500, 90]), ("observe", 4, 4, 64, 7, 7, [257, 2100, 33]),
    ("observe", 8, 2, 128, 24, 300, [700, 300, 2100])])
def test_infinite_keys_weigh_nothing(dtype, fn, Hq, Hkv, d, bs, T, lens):
    # keys with an infinite element whose logits are -inf for every query that sees them, one of them seen by
    # half of the queries alone; the other elements of the queries hold values that one bf16 holds, and zeros' tails
    print(f"\n[case] infinite keys {fn} {dtype} Hq={Hq} Hkv={Hkv} d={d} T={T}", flush=True)
    rng = np.random.default_rng(Hq * 3 + d + T)
    c = Cache(rng, "rows", dtype, Hq, Hkv, d, bs, lens)
    for s, n in enumerate(lens):
        put_key(c, s, n // 3, 5, np.inf)
        put_key(c, s, n // 2, 6, -np.inf)
        put_key(c, s, n - 1 - T // 2, 37, np.inf)
    spoil_the_rest(c)
    q = queries(rng, c, len(lens), T)
    q[..., 5] = -q[..., 5].abs() - 0.01
    q[..., 6] = q[..., 6].abs() + 0.01
    q[..., 37] = -1.0                                  # (one bf16 term holds it: the others are 0)
    seqs = [2, 0, 1]
    assert check(c, fn, seqs, q, T, 1, max(lens)) < 1


FORMS = [(fn, T, kind, dtype)
         for fn, T in (("count", 1), ("q4", 1), ("q4", 5), ("q4", 40), ("observe", 5), ("observe", 90))
         for kind, dtype in KINDS if fn != "q4" or kind == "q4"]


@pytest.mark.parametrize("fn,T,kind,dtype", FORMS)
def test_nothing_past_the_sequences_enters(fn, T, kind, dtype):
    rng = np.random.default_rng(T)
    lens = [270, 1, 700, 33]
    c = Cache(rng, kind, dtype, 8, 2, 64, 16, lens)
    spoil_the_rest(c)
    assert check(c, fn, [3, 1, 0, 2], queries(rng, c, 4, T), T, 1, 700) < 1


@pytest.mark.parametrize("fn,T,kind,dtype", FORMS + [("observe", 300, "rows", "bf16"), ("observe", 300, "q4", "f32"),
                                                     ("q4", 300, "q4", "bf16"), ("q4", 300, "q4", "f32")])
def test_a_query_of_no_weights(fn, T, kind, dtype):
    # one query whose every logit is -inf, the others as ever: it has a zero row and adds nothing
    print(f"\n[case] no weights {fn} {kind} {dtype} T={T}", flush=True)
    rng = np.random.default_rng(T)
    lens = [270, 1, 2700, 33]
    c = Cache(rng, kind, dtype, 8, 2, 64, 16, lens)
    if kind == "q4":                                   # element 9 of every key: the code of 1
        for codes in (c.host["k"], c.dev["k"]):
            codes[..., 4] = (codes[..., 4] & 15) | (2 << 4)
    else:
        c.host["k"][..., 9] = c.dev["k"][..., 9] = 1.0
    q = queries(rng, c, 4, T)
    q[0, 1, T // 2, 3, 9] = q[0, 3, T // 2, 5, 9] = q[0, 0, T - 1, 0, 9] = -np.inf
    seqs = [3, 0, 1, 2]
    assert check(c, fn, seqs, q, T, 1, 2700) < 1
    if fn != "observe":
        c = Cache(np.random.default_rng(1), kind, dtype, 8, 2, 64, 16, [40])
        assert not run(c, fn, [5], q[:, :1], T, 1, 40).any()               # (no sequence: zeros too)


@pytest.mark.parametrize("value", [np.inf, np.nan])
@pytest.mark.parametrize("fn,T,kind,dtype", FORMS)
def test_a_query_of_nan(fn, T, kind, dtype, value):
    # a logit of +inf or NaN: that query's row is NaN and the weights it gives, no others
    print(f"\n[case] NaN {fn} {kind} {dtype} T={T} {value}", flush=True)
    lens = [270, 1, 2700, 33]
    c = Cache(np.random.default_rng(T), kind, dtype, 8, 2, 64, 16, lens)
    if kind == "q4":
        for codes in (c.host["k"], c.dev["k"]):
            codes[..., 4] = (codes[..., 4] & 15) | (2 << 4)
    else:
        c.host["k"][..., 9] = c.dev["k"][..., 9] = 1.0
    q = queries(np.random.default_rng(T + 1), c, 4, T)
    seqs, at = [3, 0, 1, 2], {0: (T - 1, 0), 1: (T // 2, 3), 3: (T // 2, 5)}
    for j, (t, hq) in at.items():
        q[0, j, t, hq, 9] = value
    got = run(c, fn, seqs, q, T, 1, 2700)
    w = c.w[0].cpu().numpy()
    for j, s in enumerate(seqs):
        t, hq = at.get(j, (0, None))
        n, seen = lens[s], lens[s] - T + t + 1
        if got is not None:
            want = np.zeros(got.shape[2:4], dtype=bool)
            if hq is not None and seen > 0:
                want[t, hq] = True
            assert np.array_equal(np.isnan(got[0, j]), np.broadcast_to(want[..., None], got.shape[2:])), j
        if fn != "q4":
            want = np.zeros((n, 2), dtype=bool)
            if hq is not None:
                want[:max(seen, 0), hq // 4] = True
            pos = np.arange(n)
            assert np.array_equal(np.isnan(w[c.table[s][pos // 16], :, pos % 16]), want), j
