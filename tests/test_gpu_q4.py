"""The cache held in 4 bits (include/kara_q4.h) against fp64 numpy: appended
codes, scales, lengths and status bits exactly, rows read back exactly, and
attention within a bound counted from its roundings."""
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


def _awkward(rng, shape, dtype):
    """Rows of many magnitudes: ties, zeros of both signs, blocks of one value,
    the type's largest and smallest."""
    x = rng.standard_normal(shape) * np.exp2(rng.integers(-12, 12, shape[:-1] + (1,)))
    flat = x.reshape(-1, 32)
    n = len(flat)
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0])
    for i in range(0, n, 7):
        flat[i] = rng.choice(np.concatenate([grid, -grid, oc.MAGNITUDES]), 32) * 2.0 ** float(rng.integers(-20, 20))
    flat[1::11] = 0.0
    flat[2::13] = -0.0
    flat[3::17] *= 1e-38
    flat[4::19] = rng.choice([3.3e38, -3.3e38, 1e38, 1e30, 0.0], flat[4::19].shape)
    flat[5::23] = 0.0
    flat[5::23, 9] = 7.0000005          # past 7 units of the smaller scale (fp32), or a tie (bf16)
    t = torch.from_numpy(x.astype(np.float32)).to(cc.DT[dtype])
    return t, t.double().numpy()


@pytest.mark.parametrize("dtype,Hkv,d,bs,n_new,layers", [
    ("bf16", 8, 128, 16, 1, 1), ("bf16", 8, 128, 16, 333, 2), ("f32", 1, 64, 24, 50, 3), ("bf16", 3, 64, 7, 97, 1),
    ("f32", 5, 128, 256, 130, 1), ("bf16", 1, 128, 1, 40, 1), ("f32", 2, 128, 16, 1, 64)])
def test_append_and_read(dtype, Hkv, d, bs, n_new, layers):
    kara = _kara()
    print(f"\n[case] append {dtype} Hkv={Hkv} d={d} bs={bs} new={n_new} layers={layers}", flush=True)
    rng = np.random.default_rng(n_new * d + bs)
    lens = np.array([0, 5, 100, 33], dtype=np.int32)
    max_blocks = -(-(100 + n_new) // bs)
    table, pages, _ = cc.table_for(rng, lens + n_new, bs, max_blocks)
    seqs = np.array([2, 0, 3], dtype=np.int32)                     # sequence 1 is idle
    p = cc.params(Hkv, Hkv, d, bs, pages, max_blocks, len(lens), dtype)
    shape = (layers, pages, Hkv, bs)
    before = {x: rng.integers(0, 256, shape + (d // w,), dtype=np.uint8) for x, w in
              (("k", 2), ("v", 2), ("ks", 32), ("vs", 32))}
    pools = {x: cc.gpu(a) for x, a in before.items()}
    new, new64 = {}, {}
    for x in ("k", "v"):
        new[x], new64[x] = _awkward(rng, (layers, len(seqs), n_new, Hkv, d), dtype)
    lists = [list(pools[x].unbind(0)) for x in ("k", "v", "ks", "vs")]
    bt, sl, sq = cc.gpu(table), cc.gpu(lens), cc.gpu(seqs)
    status = torch.full((len(seqs),), 77, dtype=torch.int32, device="cuda")
    kara.q4_append(p, sq, new["k"].cuda(), new["v"].cuda(), *lists, bt, sl, status)
    torch.cuda.synchronize()
    assert status.tolist() == [0] * len(seqs)
    after = lens.copy()
    after[seqs] += n_new
    assert sl.tolist() == after.tolist()
    want = {x: a.copy() for x, a in before.items()}
    for x in ("k", "v"):
        codes, scales = oc.q4_quantize(new64[x])
        for j, s in enumerate(seqs):
            at = lens[s] + np.arange(n_new)
            for l in range(layers):
                want[x][l, table[s][at // bs], :, at % bs] = codes[l, j]
                want[x + "s"][l, table[s][at // bs], :, at % bs] = scales[l, j]
    for x in before:
        assert np.array_equal(pools[x].cpu().numpy(), want[x]), x    # all else untouched
    # read back: from before the start to past the end of every sequence
    start, n_rows = after - n_new - 3, n_new + 9
    outs = [torch.full((layers, len(seqs), n_rows, Hkv, d), 9.0, dtype=cc.DT[dtype], device="cuda") for _ in range(2)]
    kara.q4_read(p, sq, cc.gpu(start.astype(np.int32)), n_rows, *lists, bt, sl, *outs)
    for x, got in zip(("k", "v"), outs):
        got = got.double().cpu().numpy()
        for j, s in enumerate(seqs):
            for i in range(n_rows):
                pos = start[s] + i
                if 0 <= pos < after[s]:
                    page, slot = table[s][pos // bs], pos % bs
                    ref = oc.q4_values(want[x][:, page, :, slot], want[x + "s"][:, page, :, slot])
                    sane = np.repeat((want[x + "s"][:, page, :, slot] >= 2) & (want[x + "s"][:, page, :, slot] <= 252), 32, axis=-1)
                    assert np.array_equal(got[:, j, i][sane], ref[sane]), (x, s, i)   # (random bytes before: any scale)
                else:
                    assert not got[:, j, i].any(), (x, s, i)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_reports_what_is_not_finite(dtype):
    kara = _kara()
    rng = np.random.default_rng(3)
    d, Hkv, bs, n_new = 64, 2, 16, 20
    lens = np.array([3, 3, 3], dtype=np.int32)
    table, pages, _ = cc.table_for(rng, lens + n_new, bs, 2)
    p = cc.params(2, Hkv, d, bs, pages, 2, 3, dtype)
    pools = [torch.zeros((pages, Hkv, bs, d // w), dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
    x = rng.standard_normal((1, 3, n_new, Hkv, d)).astype(np.float32)
    x[0, 1, 4, 1, 7] = np.nan
    x[0, 1, 5, 0, 40] = -np.inf
    x[0, 1, 6, 0, :32] = np.inf                       # nothing finite in the block
    x = torch.from_numpy(x).to(cc.DT[dtype])
    status = torch.empty(3, dtype=torch.int32, device="cuda")
    sl = cc.gpu(lens)
    kara.q4_append(p, cc.gpu(np.array([0, 1, 2], dtype=np.int32)), x.cuda(), torch.zeros_like(x).cuda(),
                   *[[t] for t in pools], cc.gpu(table), sl, status)
    assert status.tolist() == [0, kara.SEQ_NONFINITE, 0] and sl.tolist() == (lens + n_new).tolist()
    codes, scales = oc.q4_quantize(x[0].double().numpy())
    for s in range(3):
        assert np.array_equal(cc.rows_of(pools[0].cpu().numpy(), table, s, 23, bs)[3:], codes[s])
        assert np.array_equal(cc.rows_of(pools[2].cpu().numpy(), table, s, 23, bs)[3:], scales[s])
    back = oc.q4_values(codes, scales)
    assert back[1, 4, 1, 7] == 0 and back[1, 5, 0, 40] < 0 and (back[1, 6, 0, :32] > 0).all() and np.isfinite(back).all()


def test_append_leaves_flagged_sequences():
    kara = _kara()
    rng = np.random.default_rng(4)
    d, Hkv, bs, n_new = 128, 2, 16, 40
    lens = np.array([10, 10, 10, 20, 10], dtype=np.int32)
    table, pages, _ = cc.table_for(rng, lens + n_new, bs, 4)
    table[1, 2] = pages                                # out of the pool
    table[2, 3] = -1
    lens[3] = 30                                       # 70 tokens pass the table's 64
    p = cc.params(2, Hkv, d, bs, pages, 4, 5, "bf16")
    seqs = np.array([1, 2, 3, 4, 4, -1, 5, 0], dtype=np.int32)
    pools = [torch.full((pages, Hkv, bs, d // w), 3, dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
    x = torch.randn((1, len(seqs), n_new, Hkv, d), dtype=torch.bfloat16, device="cuda")
    status = torch.empty(len(seqs), dtype=torch.int32, device="cuda")
    sl = cc.gpu(lens)
    kara.q4_append(p, cc.gpu(seqs), x, x, *[[t] for t in pools], cc.gpu(table), sl, status)
    dup = kara.SEQ_DUP_TRIGGER
    assert status.tolist() == [kara.SEQ_BAD_PAGE, kara.SEQ_BAD_PAGE, kara.SEQ_BAD_WINDOW, dup, dup, kara.SEQ_BAD_INDEX,
                               kara.SEQ_BAD_INDEX, 0]
    want = lens.copy()
    want[0] += n_new
    assert sl.tolist() == want.tolist()
    for t in pools:
        a = t.cpu().numpy()
        for page in set(range(pages)) - set(table[0][:4].tolist()):
            assert (a[page] == 3).all()


CASES = [
    # dtype, Hq, Hkv, d, bs, T, layers
    ("bf16", 32, 8, 128, 16, 1, 2), ("bf16", 40, 8, 128, 16, 1, 1), ("bf16", 4, 4, 64, 24, 1, 1),
    ("bf16", 16, 1, 64, 16, 1, 1), ("f32", 8, 2, 128, 16, 1, 1), ("f32", 16, 2, 64, 7, 3, 1),
    ("bf16", 34, 2, 128, 16, 1, 1),                        # 17 heads in a group: two row tiles
    ("bf16", 8, 2, 128, 256, 5, 2), ("bf16", 8, 8, 64, 16, 13, 1), ("f32", 6, 2, 128, 16, 40, 1),
    ("bf16", 8, 2, 128, 16, 150, 1), ("bf16", 16, 8, 64, 24, 300, 1), ("bf16", 3, 1, 128, 1, 700, 1),
]


def attention_case(dtype, Hq, Hkv, d, bs, T, layers, lens, max_len, seed=0, scale=0.0, n_extra=1):
    """Runs q4_attention over random caches; returns (worst error / bound, out)."""
    kara = _kara()
    rng = np.random.default_rng(seed + Hq * 131 + d + T)
    lens = np.asarray(lens, dtype=np.int32)
    max_blocks = -(-int(max(lens.max(), max_len)) // bs)
    table, pages, _ = cc.table_for(rng, lens, bs, max_blocks)
    seqs = rng.permutation(len(lens)).astype(np.int32)
    seqs = np.concatenate([seqs, [len(lens)] * n_extra]).astype(np.int32)      # and an index out of range
    p = cc.params(Hq, Hkv, d, bs, pages, max_blocks, len(lens), dtype, scale)
    host = {x: [cc.random_q4(rng, (pages, Hkv, bs), d) for _ in range(layers)] for x in ("k", "v")}
    lists = [[cc.gpu(c[0]) for c in host["k"]], [cc.gpu(c[0]) for c in host["v"]],
             [cc.gpu(c[1]) for c in host["k"]], [cc.gpu(c[1]) for c in host["v"]]]
    q = torch.from_numpy(rng.standard_normal((layers, len(seqs), T, Hq, d)).astype(np.float32)).to(cc.DT[dtype])
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    need = kara.q4_attention_workspace_size(p, len(seqs), layers, T, max_len)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if need else None
    kara.q4_attention(p, cc.gpu(seqs), T, q.cuda(), *lists, cc.gpu(table), cc.gpu(lens), max_len, out, ws)
    got = out.double().cpu().numpy()
    sc = scale or 1 / np.sqrt(d)
    worst = 0.0
    for l in range(layers):
        for j, s in enumerate(seqs):
            n = int(lens[s]) if s < len(lens) else 0
            if n == 0 or n > max_len:
                assert not got[l, j].any(), (l, j, n)
                continue
            k, v = (oc.q4_values(cc.rows_of(host[x][l][0], table, s, n, bs), cc.rows_of(host[x][l][1], table, s, n, bs))
                    for x in ("k", "v"))
            q64 = q[l, j].double().numpy()
            ref, mass, _ = oc.attend(q64, k, v, sc)
            delta = cc.logit_error(q64, k, sc, 1 if dtype == "bf16" else 3)
            bound = cc.attention_bound(ref, mass, delta, n, dtype, dtype == "bf16")
            if T > n:
                assert not got[l, j, :T - n].any()
            worst = max(worst, float((np.abs(got[l, j] - ref) / bound).max()))
    return worst, out


@pytest.mark.parametrize("dtype,Hq,Hkv,d,bs,T,layers", CASES)
def test_attention(dtype, Hq, Hkv, d, bs, T, layers):
    print(f"\n[case] attention {dtype} Hq={Hq} Hkv={Hkv} d={d} bs={bs} T={T}", flush=True)
    lens = [1, 31, 32, 33, 0, 255, 256, 257, 700, 900]
    worst, _ = attention_case(dtype, Hq, Hkv, d, bs, T, layers, lens, 800)     # 900 is over max_len
    print("worst error / bound", worst)
    assert worst < 1


@pytest.mark.parametrize("T", [1, 64])
def test_attention_one_split(T):
    # no sequence over the shortest split: no workspace, outputs written at once
    worst, _ = attention_case("bf16", 8, 2, 128, 16, T, 1, [1, 0, 200, 256, 17], 256)
    assert worst < 1


def test_attention_long_and_scaled():
    # a launch of many workgroups takes longer splits; a scale of the caller's
    worst, _ = attention_case("bf16", 8, 8, 64, 16, 1, 4, [5000, 1, 1025, 4999] + [40] * 60, 5000, scale=0.3)
    assert worst < 1


def test_attention_repeats_its_bits():
    a = attention_case("bf16", 32, 8, 128, 16, 4, 1, [700, 33, 1500], 1500)[1]
    b = attention_case("bf16", 32, 8, 128, 16, 4, 1, [700, 33, 1500], 1500)[1]
    assert torch.equal(a, b)


def test_far_rows():
    # codes past 4 GiB and 2^26 rows: offsets in 64 bits
    kara = _kara()
    d, Hkv, bs, n = 128, 8, 256, 300
    pages = (1 << 32) // (d // 2 * Hkv * bs) + 40
    p = cc.params(16, Hkv, d, bs, pages, 2, 1, "bf16")
    rng = np.random.default_rng(9)
    pools = [torch.empty((pages, Hkv, bs, d // w), dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
    table = np.array([[pages - 1, pages - 30]], dtype=np.int32)
    bt, sl = cc.gpu(table), cc.gpu(np.zeros(1, dtype=np.int32))
    x = {a: torch.from_numpy(rng.standard_normal((1, 1, n, Hkv, d)).astype(np.float32)).bfloat16() for a in "kv"}
    status = torch.empty(1, dtype=torch.int32, device="cuda")
    sq = cc.gpu(np.zeros(1, dtype=np.int32))
    lists = [[t] for t in pools]
    kara.q4_append(p, sq, x["k"].cuda(), x["v"].cuda(), *lists, bt, sl, status)
    assert status.item() == 0
    val = {a: oc.q4_values(*oc.q4_quantize(x[a][0, 0].double().numpy())) for a in "kv"}
    out = [torch.empty((1, 1, n, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kara.q4_read(p, sq, cc.gpu(np.zeros(1, dtype=np.int32)), n, *lists, bt, sl, *out)
    for a, t in zip("kv", out):
        assert np.array_equal(t[0, 0].double().cpu().numpy(), val[a])
    for T in (1, 128):
        q = torch.from_numpy(rng.standard_normal((1, 1, T, 16, d)).astype(np.float32)).bfloat16()
        o = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        ws = torch.empty(kara.q4_attention_workspace_size(p, 1, 1, T, n), dtype=torch.uint8, device="cuda")
        kara.q4_attention(p, sq, T, q.cuda(), *lists, bt, sl, n, o, ws)
        ref, mass, _ = oc.attend(q[0, 0].double().numpy(), val["k"], val["v"], 1 / np.sqrt(d))
        delta = cc.logit_error(q.double().numpy(), val["k"], 1 / np.sqrt(d))
        bound = cc.attention_bound(ref, mass, delta, n, "bf16", True)
        assert (np.abs(o[0, 0].double().cpu().numpy() - ref) < bound).all()


@pytest.mark.parametrize("dtype,Hq,Hkv,d,bs,T", [
    ("bf16", 32, 8, 128, 16, 20), ("bf16", 32, 8, 128, 16, 40), ("bf16", 12, 6, 64, 7, 90), ("f32", 32, 8, 128, 16, 20),
    ("f32", 16, 8, 64, 24, 60), ("bf16", 32, 8, 64, 16, 140), ("f32", 32, 8, 128, 16, 100)])
def test_attention_of_many_rows_in_larger_launches(dtype, Hq, Hkv, d, bs, T):
    # enough row blocks that keys are not split: four waves a workgroup, then eight
    lens = [1, 19, 20, 64, 65, 300, 0, 129, 700, 400, 128, 333, 90, 41, 512, 299]
    worst, _ = attention_case(dtype, Hq, Hkv, d, bs, T, 1, lens, 650)       # 700 is over max_len
    print("worst error / bound", worst)
    assert worst < 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_append_reports_and_leaves(dtype):
    # the reports and refusals of a few tokens, for an append of many
    kara = _kara()
    rng = np.random.default_rng(6)
    d, Hkv, bs, n_new, mb = 64, 3, 16, 500, 36
    lens = np.array([10, 3, 20, 10, 10, 0], dtype=np.int32)
    table, pages, _ = cc.table_for(rng, lens + n_new, bs, mb)
    table[2, 20] = pages
    lens[3] = mb * bs - n_new + 1                     # one token past the table
    p = cc.params(Hkv, Hkv, d, bs, pages, mb, len(lens), dtype)
    seqs = np.array([5, 2, 1, 3, 4, 4, 6, 0], dtype=np.int32)
    x = rng.standard_normal((1, len(seqs), n_new, Hkv, d)).astype(np.float32)
    x[0, 2, 499, 2, 63] = np.nan                      # the last element of a sequence
    x[0, 7, 250, 0, 0] = np.inf
    x[0, 1, 3, 0, 0] = np.nan                         # (of one that is left)
    x = torch.from_numpy(x).to(cc.DT[dtype])
    pools = [torch.full((pages, Hkv, bs, d // w), 3, dtype=torch.uint8, device="cuda") for w in (2, 2, 32, 32)]
    status = torch.empty(len(seqs), dtype=torch.int32, device="cuda")
    sl = cc.gpu(lens)
    kara.q4_append(p, cc.gpu(seqs), torch.zeros_like(x).cuda(), x.cuda(), *[[t] for t in pools], cc.gpu(table), sl, status)
    dup, odd = kara.SEQ_DUP_TRIGGER, kara.SEQ_NONFINITE
    assert status.tolist() == [0, kara.SEQ_BAD_PAGE, odd, kara.SEQ_BAD_WINDOW, dup, dup, kara.SEQ_BAD_INDEX, odd]
    want = lens.copy()
    want[[5, 1, 0]] += n_new
    assert sl.tolist() == want.tolist()
    codes, scales = oc.q4_quantize(x[0].double().numpy())
    touched = set()
    for j, s in ((0, 5), (2, 1), (7, 0)):
        n = int(want[s])
        touched |= set(table[s][:-(-n // bs)].tolist())
        assert np.array_equal(cc.rows_of(pools[1].cpu().numpy(), table, s, n, bs)[lens[s]:], codes[j])
        assert np.array_equal(cc.rows_of(pools[3].cpu().numpy(), table, s, n, bs)[lens[s]:], scales[j])
    for t in pools:
        assert (t.cpu().numpy()[sorted(set(range(pages)) - touched)] == 3).all()


@pytest.mark.parametrize("d,T", [(128, 80), (64, 300)])
def test_long_sums_in_fp32(d, T):
    # fp32, many rows over 8000 keys: 125 chunks of 64 keys are added to the output and to
    # the sum of weights, each addition off by half a step at most, 2^-24 / sqrt(3) of the
    # running sum on average: sqrt(2 * 125 / 3) 2^-24 = 5.4e-7 of the result (root mean
    # square); the logits' own roundings average out over the keys.  1e-6 at most.
    kara = _kara()
    rng = np.random.default_rng(d)
    n, Hq, Hkv, bs = 8000, 2, 1, 16
    table, pages, _ = cc.table_for(rng, [n], bs, n // bs)
    p = cc.params(Hq, Hkv, d, bs, pages, n // bs, 1, "f32")
    host = {x: cc.random_q4(rng, (pages, Hkv, bs), d) for x in "kv"}
    lists = [[cc.gpu(host[x][i])] for i in (0, 1) for x in "kv"]
    q = torch.from_numpy(rng.standard_normal((1, 1, T, Hq, d)).astype(np.float32)) / 8
    out = torch.empty(q.shape, device="cuda")
    ws = torch.empty(kara.q4_attention_workspace_size(p, 1, 1, T, n), dtype=torch.uint8, device="cuda")
    seqs = cc.gpu(np.zeros(1, dtype=np.int32))
    # (one listing a copy: 300 of them are enough that keys are not split)
    many = 300
    outs = torch.empty((1, many, T, Hq, d), device="cuda")
    ws_many = torch.empty(kara.q4_attention_workspace_size(p, many, 1, T, n), dtype=torch.uint8, device="cuda")
    bt, sl = cc.gpu(table), cc.gpu(np.array([n], dtype=np.int32))
    kara.q4_attention(p, seqs, T, q.cuda(), *lists, bt, sl, n, out, ws)
    kara.q4_attention(p, seqs.repeat(many), T, q.cuda().expand(outs.shape).contiguous(), *lists, bt, sl, n, outs, ws_many)
    k, v = (oc.q4_values(cc.rows_of(host[x][0], table, 0, n, bs), cc.rows_of(host[x][1], table, 0, n, bs)) for x in "kv")
    ref = oc.attend(q[0, 0].double().numpy(), k, v, 1 / np.sqrt(d))[0]
    for got in (out[0, 0], outs[0, 0], outs[0, many - 1]):
        err = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
        print("error", err)
        assert err < 1e-6
