"""The serving operators as they are used together: prompts and decoding steps whose
tokens are turned on their way into a cache of rows or of 8-bit codes and attended over
in a window, its dropped pages taken back; on other streams, captured and replayed, and
at the far end of large pools."""
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


def _kara():
    from paper_2607_01237_amd import kara
    return kara


THETA = 1e4


class Program:
    """Two layers, three sequences: the second layer's tokens follow the first's."""

    def __init__(self, cache, dtype="bf16", window=40, sink=3, d=64, bs=16, max_blocks=30, pages=40, seed=0):
        self.k = _kara()
        self.cache, self.dtype, self.window, self.sink, self.d, self.bs = cache, dtype, window, sink, d, bs
        self.layers, self.n, self.Hq, self.Hkv = 2, 3, 8, 2
        self.rng = np.random.default_rng(seed)
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.free = self.rng.permutation(pages).tolist()
        self.table = np.full((self.n, max_blocks), -1, dtype=np.int32)
        self.lens = np.zeros(self.n, dtype=np.int32)
        self.rot = np.array([0, 1000, 77], dtype=np.int32)
        self.p = cc.params(self.Hq, self.Hkv, d, bs, pages, max_blocks, self.n, dtype)
        self.rope = self.k.make_rope(theta=THETA)
        shape = (self.layers, pages, self.Hkv, bs, d)
        if cache == "q8":     # what was there before may be anything
            self.pool = {x: torch.full(shape, 255, dtype=torch.uint8, device="cuda") for x in "kv"}
            self.scale = {x: torch.full(shape[:3], 255, dtype=torch.uint8, device="cuda") for x in "kv"}
        else:
            self.pool = {x: torch.full(shape, float("nan"), dtype=cc.DT[dtype], device="cuda") for x in "kv"}
            self.scale = None
        self.bt, self.sl, self.rp = cc.gpu(self.table), cc.gpu(self.lens), cc.gpu(self.rot)
        self.seqs = cc.gpu(np.array([2, 0, 1], dtype=np.int32))
        self.status = torch.full((self.n,), 9, dtype=torch.int32, device="cuda")
        self.max_len = max_blocks * bs
        need = max(self.k.window_attention_workspace_size(self.p, self.n, 1, T, window, sink, self.max_len) for T in (1, 9, 50, 64, 100))
        self.ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")

    def randn(self, *shape):
        return torch.randn(shape, generator=self.gen, device="cuda").to(cc.DT[self.dtype])

    def tokens(self, T):
        return {x: self.randn(self.layers, self.n, T, h, self.d) for x, h in (("q", self.Hq), ("k", self.Hkv), ("v", self.Hkv))}

    def grow(self, T):
        """Maps the blocks of T more tokens; gives back those that no query will see again."""
        for s in range(self.n):
            if self.window:
                last = int(self.lens[s]) - self.window + 1       # the next query's first key, but for the sinks
                for b in range(-(-self.sink // self.bs), max(0, last // self.bs)):
                    if self.table[s, b] >= 0:
                        self.free.insert(0, int(self.table[s, b]))
                        self.table[s, b] = -1
            for b in range(-(-int(self.lens[s]) // self.bs), -(-(int(self.lens[s]) + T) // self.bs)):
                self.table[s, b] = self.free.pop()
        self.bt.copy_(torch.from_numpy(self.table))

    def step(self, x, out, q_out, stream=None):
        """One step of all layers, each as its own calls."""
        T = x["q"].shape[2]
        for l in range(self.layers):
            kw = {} if self.scale is None else dict(k_scales=[self.scale["k"][l]], v_scales=[self.scale["v"][l]])
            pools = [self.pool["k"][l]], [self.pool["v"][l]]
            self.k.rope_append(self.p, self.rope, self.seqs, x["k"][l:l + 1], x["v"][l:l + 1], *pools, self.bt, self.sl,
                               self.status, rope_pos=self.rp, q=x["q"][l:l + 1], q_out=q_out[l:l + 1], counted=l > 0,
                               stream=stream, **kw)
            self.k.window_attention(self.p, self.seqs, T, self.window, self.sink, q_out[l:l + 1], *pools, self.bt, self.sl,
                                    self.max_len, out[l:l + 1], self.ws, stream=stream, **kw)

    def counted(self, T):
        self.lens += T
        self.rot += T


@pytest.mark.parametrize("cache,dtype,window,sink", [("q8", "bf16", 40, 3), ("rows", "bf16", 40, 3), ("q8", "f32", 33, 0),
                                                     ("rows", "f32", 40, 20), ("q8", "bf16", 0, 0)])
def test_prompts_and_steps(cache, dtype, window, sink):
    pr = Program(cache, dtype, window, sink, max_blocks=30, pages=100 if window == 0 else 40)
    kept = {(l, s): [np.zeros((0, pr.Hkv, pr.d)) for _ in range(2)] for l in range(pr.layers) for s in range(pr.n)}
    for T in [50] + [1] * 45 + [64, 1, 9, 1]:
        pr.grow(T)
        x = pr.tokens(T)
        out, q_out = torch.full_like(x["q"], 7.0), torch.empty_like(x["q"])
        pr.step(x, out, q_out)
        pr.counted(T)
        assert not pr.status.any() and pr.sl.tolist() == pr.lens.tolist() and pr.rp.tolist() == pr.rot.tolist()
        pools = {y: pr.pool[y].cpu() for y in "kv"}
        for l in range(pr.layers):
            for j, s in enumerate(pr.seqs.tolist()):
                n = int(pr.lens[s])
                pos = pr.rot[s] - T + np.arange(T)
                q64 = q_out[l, j].double().cpu().numpy()
                want_q = ks.turn(x["q"][l, j].double().cpu().numpy(), pos, pr.d, theta=THETA)
                half_step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
                assert (np.abs(q64 - want_q) <= (half_step + 2.0 ** -19) * (np.abs(want_q) + 16)).all()
                # what the cache holds of the positions still mapped; the others as they were
                new = []
                for y in "kv":
                    rows = np.concatenate([kept[l, s]["kv".index(y)], np.zeros((T, pr.Hkv, pr.d))])
                    at = np.flatnonzero(pr.table[s][np.arange(n) // pr.bs] >= 0)
                    page, slot = pr.table[s][at // pr.bs], at % pr.bs
                    if cache == "q8":
                        rows[at] = ks.q8_values(pools[y][l].numpy()[page, :, slot],
                                                pr.scale[y][l].cpu().numpy()[page][:, :, None])
                    else:
                        rows[at] = pools[y][l].double().numpy()[page, :, slot]
                    new.append(rows)
                kept[l, s] = new
                turned = ks.turn(x["k"][l, j].double().cpu().numpy(), pos, pr.d, theta=THETA)
                step = (2.0 ** -4 if cache == "q8" else half_step) + 2.0 ** -19
                assert (np.abs(new[0][n - T:] - turned) <= step * (np.abs(turned) + 2.0 ** -6) + 2.0 ** -18 * 16).all()
                scale = 1 / np.sqrt(pr.d)
                ref, mass = ks.attend(q64, *new, scale, window, sink)
                delta = cc.logit_error(q64, new[0], scale, 1 if dtype == "bf16" else 3)
                bound = cc.attention_bound(ref, mass, delta, n, dtype, dtype == "bf16")
                assert (np.abs(out[l, j].double().cpu().numpy() - ref) <= bound).all(), (T, n, l, s)


@pytest.mark.parametrize("cache", ["q8", "rows"])
def test_on_another_stream(cache):
    # everything queued on a side stream, behind work that takes a while: the bits of the main one
    outs = []
    for stream in (None, torch.cuda.Stream()):
        pr = Program(cache)
        steps = [pr.tokens(T) for T in (50, 1, 64, 1)]
        pr.grow(116)
        got = []
        res = [(torch.empty_like(x["q"]), torch.empty_like(x["q"])) for x in steps]
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(stream):
                big = torch.randn(4096, 4096, device="cuda")
                for _ in range(5):
                    big = big @ big * 1e-2
        for x, (out, q_out) in zip(steps, res):
            pr.step(x, out, q_out, stream=stream)
            got += [out, q_out]
        torch.cuda.synchronize()
        assert not pr.status.any()
        outs.append(got + [pr.sl, pr.rp, pr.status] + [t.view(torch.uint8) for t in pr.pool.values()])
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_two_programs_at_once():
    # on two streams, each with its own workspace, in turns that overlap: the bits of one alone
    def fresh(seed):
        pr = Program("q8", seed=seed, pages=100)
        pr.grow(300)
        steps = [pr.tokens(T) for T in (64, 1, 1, 100, 1, 64)]
        return pr, steps, [(torch.empty_like(x["q"]), torch.empty_like(x["q"])) for x in steps]

    alone = [fresh(1), fresh(2)]
    for pr, steps, res in alone:
        for x, r in zip(steps, res):
            pr.step(x, *r)
    torch.cuda.synchronize()
    both = [fresh(1), fresh(2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(6):
        for (pr, steps, res), stream in zip(both, streams):
            pr.step(steps[i], *res[i], stream=stream)
    torch.cuda.synchronize()
    for (p1, _, r1), (p2, _, r2) in zip(alone, both):
        for a, b in zip(r1, r2):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.equal(p1.sl, p2.sl) and all(torch.equal(p1.pool[y], p2.pool[y]) for y in "kv")


@pytest.mark.parametrize("cache", ["q8", "rows"])
def test_captured(cache):
    # a decoding step and a prompt's chunk captured into two graphs that share a workspace,
    # replayed in turns with eager work and synchronisations between: the bits of eager calls
    def fresh():
        pr = Program(cache, pages=100)
        pr.grow(400)
        return pr, {T: pr.tokens(T) for T in (1, 64)}

    eager, x = fresh()
    pr, y = fresh()
    gen = torch.Generator(device="cuda").manual_seed(5)
    res = {T: (torch.empty_like(t["q"]), torch.empty_like(t["q"])) for T, t in y.items()}
    want = {T: (torch.empty_like(t["q"]), torch.empty_like(t["q"])) for T, t in x.items()}
    graphs = {}
    torch.cuda.synchronize()
    for T in (1, 64):
        graphs[T] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[T]):
            pr.step(y[T], *res[T])
    assert pr.sl.tolist() == [0, 0, 0]                   # captured, not run
    for turn, T in enumerate((64, 1, 1, 64, 1, 64, 64, 1)):
        for name in "qkv":
            fill = torch.randn(x[T][name].shape, generator=gen, device="cuda").to(x[T][name].dtype)
            x[T][name].copy_(fill)
            y[T][name].copy_(fill)
        if turn % 2:
            torch.cuda.synchronize()
        graphs[T].replay()
        eager.step(x[T], *want[T])
        if turn % 3 == 0:
            pr.ws.fill_(turn)                            # (nothing is kept in it between calls)
        assert torch.equal(res[T][0], want[T][0]) and torch.equal(res[T][1], want[T][1]), turn
        assert pr.sl.tolist() == eager.sl.tolist() and pr.rp.tolist() == eager.rp.tolist()
        assert all(torch.equal(pr.pool[z].view(torch.uint8), eager.pool[z].view(torch.uint8)) for z in "kv")


@pytest.mark.parametrize("cache,T", [("rows", 1), ("rows", 40), ("q8", 1), ("q8", 40), ("f32", 3)])
def test_far_end_of_large_pools(cache, T):
    # pages past the 4 GiB of bytes that 32 bits address
    kara = _kara()
    Hq, Hkv, d, bs, n = 8, 8, 128, 16, 200
    dtype = "f32" if cache == "f32" else "bf16"
    row = d * {"rows": 2, "q8": 1, "f32": 4}[cache]
    pages = (5 << 30) // (Hkv * bs * row)
    blocks = -(-(n + T) // bs)
    table = (pages - 1 - np.arange(blocks, dtype=np.int32) * 3)[None]
    table[0, 1] = 2                                       # one near the start
    p = cc.params(Hq, Hkv, d, bs, pages, blocks, 1, dtype)
    pools = [torch.zeros((pages, Hkv, bs, d), dtype=torch.uint8 if cache == "q8" else cc.DT[dtype], device="cuda")
             for _ in range(2)]
    kw = {} if cache != "q8" else {x + "_scales": [torch.zeros((pages, Hkv), dtype=torch.uint8, device="cuda")] for x in "kv"}
    sl, rp = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    seqs, status, bt = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), 7, dtype=torch.int32, device="cuda"), cc.gpu(table)
    rope = kara.make_rope(theta=THETA)
    for m in (n, T):
        k, v = (torch.randn((1, 1, m, Hkv, d), device="cuda").to(cc.DT[dtype]) for _ in range(2))
        q = torch.randn((1, 1, m, Hq, d), device="cuda").to(cc.DT[dtype])
        kara.rope_append(p, rope, seqs, k, v, [pools[0]], [pools[1]], bt, sl, status, rope_pos=rp, q=q, q_out=q, **kw)
        assert status.tolist() == [0]
    out = torch.empty_like(q)
    ws = torch.empty(max(1, kara.window_attention_workspace_size(p, 1, 1, T, 150, 5, n + T)), dtype=torch.uint8, device="cuda")
    kara.window_attention(p, seqs, T, 150, 5, q, [pools[0]], [pools[1]], bt, sl, n + T, out, ws, **kw)
    at = np.arange(n + T)
    page, slot = torch.from_numpy(table[0][at // bs]).long().cuda(), torch.from_numpy(at % bs).cuda()
    rows = []
    for x, t in zip("kv", pools):
        y = t[page, :, slot].cpu()
        rows.append(ks.q8_values(y.numpy(), kw[x + "_scales"][0][page].cpu().numpy()[:, :, None]) if cache == "q8"
                    else y.double().numpy())
    assert np.abs(rows[1]).sum((1, 2)).all()              # every position was written
    q64 = q[0, 0].double().cpu().numpy()
    ref, mass = ks.attend(q64, *rows, 1 / np.sqrt(d), 150, 5)
    delta = cc.logit_error(q64, rows[0], 1 / np.sqrt(d), 1 if dtype == "bf16" else 3)
    bound = cc.attention_bound(ref, mass, delta, n + T, dtype, dtype == "bf16")
    assert (np.abs(out[0, 0].double().cpu().numpy() - ref) <= bound).all()


@pytest.mark.parametrize("layers", [1, 2, 3, 11])
def test_layers_of_one_call(layers):
    # a call of many layers gives each the bits of a call of its own, of few tokens and of many
    kara = _kara()
    rng = np.random.default_rng(layers)
    Hq, Hkv, d, bs = 8, 4, 64, 16
    for T in (1, 5, 70):
        lens = np.array([40, 7], dtype=np.int32)
        table, pages, _ = cc.table_for(rng, lens + T, bs, 10)
        p = cc.params(Hq, Hkv, d, bs, pages, 10, 2, "bf16")
        x = {y: torch.randn((layers, 2, T, h, d), device="cuda").bfloat16() for y, h in (("q", Hq), ("k", Hkv), ("v", Hkv))}
        got = []
        for one in (False, True):
            pools = [torch.zeros((layers, pages, Hkv, bs, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.full((layers, pages, Hkv), 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
            sl, status = cc.gpu(lens), torch.full((2,), 7, dtype=torch.int32, device="cuda")
            sq, bt = cc.gpu(np.array([1, 0], dtype=np.int32)), cc.gpu(table)
            q_out, out = torch.empty_like(x["q"]), torch.empty_like(x["q"])
            ws = torch.empty(max(1, kara.window_attention_workspace_size(p, 2, layers, T, 30, 2, 160)), dtype=torch.uint8, device="cuda")
            for a, b in [(l, l + 1) for l in range(layers)] if one else [(0, layers)]:
                args = [list(t[a:b].unbind(0)) for t in pools]
                kw = dict(k_scales=list(scales[0][a:b].unbind(0)), v_scales=list(scales[1][a:b].unbind(0)))
                kara.rope_append(p, kara.make_rope(), sq, x["k"][a:b], x["v"][a:b], *args, bt, sl, status, q=x["q"][a:b],
                                 q_out=q_out[a:b], counted=a > 0, **kw)
                assert status.tolist() == [0, 0]
                kara.window_attention(p, sq, T, 30, 2, q_out[a:b], *args, bt, sl, 160, out[a:b], ws, **kw)
            got.append([q_out, sl, *pools, *scales])
            if not one:
                whole = out
        assert all(torch.equal(u, v) for u, v in zip(*got))
        # (keys may be split otherwise: the last bits of an output)
        assert (whole.float() - out.float()).abs().max() <= 2.0 ** -6


def test_prompts_of_many_lengths():
    """Calls whose long sequences' keys are split by their lengths, and calls with more workgroups than that."""
    kara = _kara()
    rng = np.random.default_rng(0)
    Hq, Hkv, d, bs = 4, 1, 64, 16
    for cache, seqs_n, T in (("q8", 6, 100), ("rows", 6, 100), ("q8", 1, 40), ("rows", 2, 300), ("q8", 130, 70), ("rows", 300, 50),
                             ("q8", 600, 33), ("f32", 3, 60)):
        dtype = "f32" if cache == "f32" else "bf16"
        lens = np.maximum(1, (rng.uniform(0, 1, seqs_n) ** 3 * 3000)).astype(np.int32)
        lens[0] = 3000
        if seqs_n > 4:
            lens[3] = T // 2                                   # shorter than its queries
        table, pages, _ = cc.table_for(rng, lens, bs, -(-3000 // bs))
        p = cc.params(Hq, Hkv, d, bs, pages, table.shape[1], seqs_n, dtype)
        if cache == "rows":
            pools = [torch.randn((pages, Hkv, bs, d), device="cuda").bfloat16() for _ in range(2)]
            values = [t.double().cpu().numpy() for t in pools]
            kw = {}
        else:
            pools = [torch.randint(0, 0x48, (pages, Hkv, bs, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
            pools = [t + 128 * torch.randint_like(t, 0, 2) for t in pools]
            scales = [torch.randint(124, 128, (pages, Hkv), dtype=torch.uint8, device="cuda") for _ in range(2)]
            values = [ks.q8_values(t.cpu().numpy(), s.cpu().numpy()[:, :, None, None]) for t, s in zip(pools, scales)]
            kw = dict(k_scales=[scales[0]], v_scales=[scales[1]])
        order = rng.permutation(seqs_n).astype(np.int32)
        q = torch.randn((1, seqs_n, T, Hq, d), device="cuda").to(cc.DT[dtype])
        out = torch.full_like(q, 7.0)
        need = kara.window_attention_workspace_size(p, seqs_n, 1, T, 0, 0, 3000)
        ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
        kara.window_attention(p, cc.gpu(order), T, 0, 0, q, [pools[0]], [pools[1]], cc.gpu(table), cc.gpu(lens), 3000, out,
                              ws[:need], **kw)
        assert (ws[need:] == 255).all()
        some = np.flatnonzero(np.isin(order, [0, 3, *rng.integers(0, seqs_n, 4)]))
        for j in some:
            s = int(order[j])
            n = int(lens[s])
            at = np.arange(n)
            k, v = (x[table[s][at // bs], :, at % bs] for x in values)
            rows = sorted({0, T - 1, max(0, T - n), *rng.integers(0, T, 6).tolist()})
            q64 = q[0, j].double().cpu().numpy()
            for t in rows:
                m = n - (T - 1 - t)
                if m <= 0:
                    assert not out[0, j, t].any()
                    continue
                ref, mass = ks.attend(q64[t:t + 1], k[:m], v[:m], 0.125)
                delta = cc.logit_error(q64[t:t + 1], k[:m], 0.125, 1 if dtype == "bf16" else 3)
                bound = cc.attention_bound(ref, mass, delta, m, dtype, dtype == "bf16")
                assert (np.abs(out[0, j, t].double().cpu().numpy() - ref[0]) <= bound[0]).all(), (cache, seqs_n, s, t)


def test_refused_on_the_host():
    kara = _kara()
    pr = Program("rows")
    x = pr.tokens(1)
    pools = [pr.pool["k"][0]], [pr.pool["v"][0]]
    args = (x["k"][:1], x["v"][:1], *pools, pr.bt, pr.sl, pr.status)
    with pytest.raises(kara.KaraError):
        kara.rope_append(pr.p, pr.rope, pr.seqs, *args, q=x["q"][:1])                    # queries without a place
    with pytest.raises(kara.KaraError):
        kara.rope_append(pr.p, kara.make_rope(dim=32, inv_freq=torch.zeros(16)), pr.seqs, *args)   # on the host
    with pytest.raises(kara.KaraError):
        kara.rope_append(pr.p, pr.rope, pr.seqs.cpu(), *args)
    with pytest.raises(kara.KaraError):
        kara.window_attention(pr.p, pr.seqs, 2, 4, 0, x["q"][:1], *pools, pr.bt, pr.sl, 64, x["q"][:1], pr.ws)   # one query
    with pytest.raises(kara.KaraError):
        kara.window_attention(pr.p, pr.seqs, 1, 4, 0, x["q"][:1], *pools, pr.bt, pr.sl, 64, torch.empty_like(x["q"][:1]),
                              pr.ws, k_scales=[torch.zeros(9999, dtype=torch.uint8, device="cuda")])
    with pytest.raises(kara.KaraError):
        kara.q8_append(pr.p, pr.seqs, x["k"][:1], x["v"][:1], *pools, None, None, pr.bt, pr.sl, pr.status)
    torch.cuda.synchronize()
    assert pr.sl.tolist() == [0, 0, 0] and pr.status.tolist() == [9, 9, 9]
