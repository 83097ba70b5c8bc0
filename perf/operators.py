"""Operators beside the compression step, each with its plain form.

Five kinds of pass:

append     tokens quantised into a cache held in 4 bits (kara.q4_append), and
           the new rows read back (kara.q4_read).
attention  causal attention of each sequence's last n_query tokens over a cache
           held in 4 bits (kara.q4_attention): decoding steps, drafted tokens,
           chunks of a prompt.
weigh      a decoding step's attention that also adds each cached token's weight
           to its accumulator (kara.evict_attention), over rows or 4 bits.
observe    the weights that a prompt's queries give, added to the accumulators
           (kara.evict_observe).
evict      the cache cut to `keep` tokens per KV head by accumulated weight
           (kara.evict_tokens): pages, tables and accumulators after it.

A cache in 4 bits holds blocks of 32 values of a row: e2m1 codes (0, .5, 1, 1.5,
2, 3, 4, 6 and a sign; the even element in the low half of a byte) and a scale
byte b, worth 2^(b - 127).  The exponent is the largest magnitude's, less two,
or one more where that magnitude is over 7 of the smaller scale's units.

Sizes are those of the workloads in kara_inputs and perf/cases.py; inputs are
N(0, 1) rows (model weights are not available), a few keys four times as large.
"""
import math

import numpy as np
import torch

own = False

_DEV = "cuda:0"

_APPEND = dict(kind="append", dtype="bf16", n_q=32, n_kv=8, d=128, seqs=8, idle=2, layers=1, len_lo=300, len_hi=4000,
               new=1, block=16)
_ATTENTION = dict(kind="attention", dtype="bf16", n_q=32, n_kv=8, d=128, seqs=8, idle=2, layers=1, len_lo=300,
                  len_hi=4000, queries=1, block=16)
_WEIGH = dict(_ATTENTION, kind="weigh", cache="rows")
_OBSERVE = dict(_ATTENTION, kind="observe", cache="rows", queries=1024)
_EVICT = dict(kind="evict", cache="rows", dtype="bf16", n_q=32, n_kv=8, d=128, seqs=8, idle=2, layers=1, len_lo=300,
              len_hi=4000, keep=1024, sink=4, recent=256, block=16)


def listed():
    return [
        # one decoding step of a small batch, one layer: all launch latency and host work
        dict(_APPEND, name="append_step"),
        # the prompts of a few requests quantised after prefill
        dict(_APPEND, name="append_prompt", seqs=4, idle=0, layers=4, len_lo=0, len_hi=90, new=4000),
        # a decoding step over 4 bits: a small batch, and a long-context one
        dict(_ATTENTION, name="attend_step"),
        dict(_ATTENTION, name="attend_long", n_q=40, seqs=96, idle=4, layers=2, len_lo=7000, len_hi=8190),
        # five drafted tokens checked at once, fp32 activations, 64-wide heads, odd lengths and pages
        dict(_ATTENTION, name="attend_drafted_f32", dtype="f32", n_q=16, n_kv=2, d=64, seqs=13, len_lo=97, len_hi=3001,
             queries=5, block=24),
        # a prompt's next chunk over what is cached
        dict(_ATTENTION, name="attend_chunk", seqs=4, idle=0, len_lo=2500, len_hi=8700, queries=512),
        # a decoding step with accumulators, over rows and over 4 bits
        dict(_WEIGH, name="weigh_rows", seqs=8),
        dict(_WEIGH, name="weigh_q4_long", cache="q4", n_q=40, seqs=64, idle=4, layers=2, len_lo=4000, len_hi=8190),
        # two whole prompts' weights; a short observation window over 4 bits
        dict(_OBSERVE, name="observe_prompt", seqs=2, idle=0, len_lo=2048, len_hi=4001, queries=2048),
        dict(_OBSERVE, name="observe_window_q4", cache="q4", n_q=16, n_kv=8, d=64, seqs=6, len_lo=700, len_hi=5003,
             queries=33, block=24),
        # caches cut to their budget: a layer of a small batch, and a large batch's layers
        dict(_EVICT, name="evict_layer"),
        dict(_EVICT, name="evict_batch", seqs=64, idle=4, layers=4, len_lo=3900, len_hi=8190, keep=3800, recent=1000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "weigh", "observe", "evict"])
    while True:
        n_q, n_kv, d = rng.choice([(32, 8, 128), (40, 8, 128), (16, 8, 64), (16, 2, 64), (8, 8, 128), (8, 1, 128)])
        lo = _log_int(rng, 20, 6000)
        c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), n_q=n_q, n_kv=n_kv, d=d,
                 seqs=_log_int(rng, 1, 96), idle=rng.randrange(0, 4), layers=_log_int(rng, 1, 8), len_lo=lo,
                 len_hi=lo + _log_int(rng, 1, 6000), block=rng.choice([16, 16, 256, 24]))
        if kind == "append":
            c.update(new=rng.choice([1, _log_int(rng, 1, 4000)]))
        elif kind == "attention":
            c.update(queries=rng.choice([1, rng.randrange(2, 9), _log_int(rng, 9, 1000)]))
        elif kind == "weigh":
            c.update(queries=1, cache=rng.choice(["rows", "q4"]))
        elif kind == "observe":
            c.update(queries=_log_int(rng, 2, 2048), cache=rng.choice(["rows", "q4"]))
        else:
            keep = _log_int(rng, 16, c["len_hi"])
            c.update(keep=keep, sink=rng.randrange(0, min(keep, 9)), recent=rng.randrange(0, max(1, keep // 2 - 8)),
                     cache=rng.choice(["rows", "rows", "q4"]))
        w = work(c)
        # (at rough rates, under the largest listed pass; the plain forms' arrays fit the card several times)
        if w["bytes"] / 4e12 + w["flops"] / 4e14 <= 5e-4 and _plain_values(c) < 2.5e9:
            return c


# ---- geometry

def _lengths(c):
    """Tokens in each sequence before the pass, the listed ones first: a fixed spread over the case's range."""
    n = c["seqs"] + c["idle"]
    lens = np.linspace(c["len_lo"], c["len_hi"], n).round().astype(np.int64) if n > 1 else np.array([c["len_hi"]])
    return np.random.default_rng(n).permutation(lens)


def _plain_values(c):
    """The most values an array of the plain form holds."""
    M = c["len_hi"] + c.get("new", 0)
    rows = c["layers"] * c["seqs"] * c["n_kv"] * M
    return rows * max(c["d"], c["n_q"] // c["n_kv"] * c.get("queries", 1))


def work(c):
    e = 4 if c["dtype"] == "f32" else 2
    lens = _lengths(c)[:c["seqs"]]
    L, S, H, G, d = c["layers"], c["seqs"], c["n_kv"], c["n_q"] // c["n_kv"], c["d"]
    q4 = d // 2 + d // 32
    if c["kind"] == "append":
        rows = L * S * H * c["new"]
        return {"bytes": 2 * rows * (2 * d * e + 2 * q4), "flops": 0}
    if c["kind"] == "evict":
        row = 2 * (q4 if c["cache"] == "q4" else d * e) + 4
        cut = lens > c["keep"]
        read = c["seqs"] * c["keep"] * 2 * d * e if c["cache"] == "q4" else 0
        return {"bytes": L * H * (int(lens[cut].sum()) * 4 + int(cut.sum()) * c["keep"] * (2 * row + 4) + read), "flops": 0}
    T = c["queries"]
    keys = int(lens.sum())
    pairs = int(sum(T * n - T * (T - 1) // 2 if n >= T else n * (n + 1) // 2 for n in lens.tolist()))
    io = L * S * T * c["n_q"] * d
    if c["kind"] == "attention":
        return {"bytes": L * H * keys * 2 * q4 + 2 * io * e, "flops": L * pairs * 4 * c["n_q"] * d}
    row = q4 if c["cache"] == "q4" else d * e
    if c["kind"] == "weigh":
        return {"bytes": L * H * keys * (2 * row + 8) + io * (e + 4), "flops": L * pairs * 4 * c["n_q"] * d}
    return {"bytes": L * H * keys * (row + 8) + io * e, "flops": L * pairs * 2 * c["n_q"] * d}


# ---- inputs

def _tables(c, seed):
    """Tables of a fragmented pool: every sequence mapped for its tokens and those the pass adds."""
    lens, bs = _lengths(c), c["block"]
    need = [-(-int(n + (c.get("new", 0) if i < c["seqs"] else 0)) // bs) for i, n in enumerate(lens)]
    pages = math.ceil(sum(need) * 1.05) + 1
    order = np.random.default_rng(seed).permutation(pages)
    table = np.full((len(lens), max(max(need), 1)), -1, dtype=np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return lens.astype(np.int32), table, pages


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(_DEV)


def prepare(c, seed):
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed))
    randn = lambda shape, t=dt: torch.randn(shape, generator=g, device=_DEV, dtype=t)  # noqa: E731
    lens, table, pages = _tables(c, seed)
    L, S, H, d, bs = c["layers"], c["seqs"], c["n_kv"], c["d"], c["block"]
    i32 = dict(dtype=torch.int32, device=_DEV)
    st = dict(case=c, pages=pages, scale=1.0 / math.sqrt(d))
    st["bt0"], st["lens0"] = _dev(table), _dev(lens)
    st["bt"], st["lens"] = st["bt0"].clone(), st["lens0"].clone()
    st["seqs"] = _dev(np.random.default_rng(seed).permutation(S).astype(np.int32))
    st["status"] = torch.zeros(S, **i32)
    # (a page more than the pool's: the plain form writes there what belongs nowhere)
    shape = (L, pages + 1, H, bs)
    if c["kind"] == "append" or c.get("cache", "q4") == "q4":
        st["k"], st["v"] = (torch.zeros(shape + (d // 2,), dtype=torch.uint8, device=_DEV) for _ in range(2))
        st["ks"], st["vs"] = (torch.full(shape + (d // 32,), 127, dtype=torch.uint8, device=_DEV) for _ in range(2))
        if c["kind"] != "append":
            for layer in range(L):
                for codes, scales in ((st["k"], st["ks"]), (st["v"], st["vs"])):
                    x = randn(shape[1:] + (d,))
                    x.mul_(torch.where(torch.rand(shape[1:] + (1,), generator=g, device=_DEV) < 0.02, 4.0, 1.0).to(dt))
                    codes[layer], scales[layer] = _quantize(x)
    else:
        st["k"], st["v"] = randn(shape + (d,)), randn(shape + (d,))
    if c["kind"] == "append":
        st["k_new"], st["v_new"] = (randn((L, S, c["new"], H, d)) for _ in range(2))
        st["k_out"], st["v_out"] = torch.empty_like(st["k_new"]), torch.empty_like(st["v_new"])
    if c["kind"] in ("weigh", "observe", "evict"):
        # eviction: weights fall off like 1 / rank, few tokens hold most, one in ten has none;
        # accumulation: the first steps, when what is added shows
        u = torch.rand(shape, generator=g, device=_DEV)
        st["weights0"] = torch.where(u < 0.1, 0.0, 0.1 / (1.0001 - u)) if c["kind"] == "evict" else u * 0.001
        del u
        st["weights"] = st["weights0"].clone()
    if c["kind"] in ("attention", "weigh", "observe"):
        st["q"] = randn((L, S, c["queries"], c["n_q"], d))
        if c["kind"] != "observe":
            st["out"] = torch.empty_like(st["q"], dtype=torch.float32 if c["kind"] == "weigh" else dt)
    if c["kind"] == "evict":
        st["kept"] = torch.empty((L, S, H, c["keep"]), **i32)
        st["freed"], st["n_freed"] = torch.empty((S, table.shape[1]), **i32), torch.empty(S, **i32)
        if c["cache"] == "q4":
            st["k_out"], st["v_out"] = (torch.empty((L, S, c["keep"], H, d), dtype=dt, device=_DEV) for _ in range(2))
            st["start"] = torch.zeros_like(st["lens"])
    st["max_len"] = int(lens.max()) + c.get("new", 0)
    if own:
        _plan(st)
    return st


def _plan(st):
    """What a program keeps beside its tensors: geometry, the layers' pools, workspaces."""
    from paper_2607_01237_amd import kara
    c = st["case"]
    L, S = c["layers"], c["seqs"]
    p = st["p"] = kara.make_params(dict(
        window=64, buffer=0, budget=16, chunk_budget=0, max_chunk_len=4, head_dim=c["d"], n_q_heads=c["n_q"],
        n_kv_heads=c["n_kv"], block_size=c["block"], num_pages=st["pages"], max_blocks_per_seq=st["bt"].shape[1],
        dtype=c["dtype"], scale=0.0, score_queries=0), S + c["idle"])
    st["kp"], st["vp"] = list(st["k"].unbind(0)), list(st["v"].unbind(0))
    st["ksp"], st["vsp"] = (list(st[x].unbind(0)) if x in st else None for x in ("ks", "vs"))
    st["wp"] = list(st["weights"].unbind(0)) if "weights" in st else None
    size = {"attention": lambda: kara.q4_attention_workspace_size(p, S, L, c["queries"], st["max_len"]),
            "weigh": lambda: kara.evict_attention_workspace_size(p, S, L, st["max_len"]),
            "observe": lambda: kara.evict_observe_workspace_size(p, S, L, c["queries"], st["max_len"]),
            "evict": lambda: kara.evict_workspace_size(p, S, L, c["keep"])}.get(c["kind"])
    if size:
        st["ws"] = torch.empty(max(1, size()), dtype=torch.uint8, device=_DEV)


# ---- one pass

def run(st):
    st["lens"].copy_(st["lens0"])
    if st["case"]["kind"] == "evict":
        st["bt"].copy_(st["bt0"])
        st["weights"].copy_(st["weights0"])
    return (_own if own else _plain)[st["case"]["kind"]](st)


def _own_append(st):
    from paper_2607_01237_amd import kara
    cache = (st["kp"], st["vp"], st["ksp"], st["vsp"], st["bt"], st["lens"])
    kara.q4_append(st["p"], st["seqs"], st["k_new"], st["v_new"], *cache, st["status"])
    kara.q4_read(st["p"], st["seqs"], st["lens0"], st["case"]["new"], *cache, st["k_out"], st["v_out"])
    return dict(k=st["k_out"], v=st["v_out"], lens=st["lens"], status=st["status"])


def _own_attention(st):
    from paper_2607_01237_amd import kara
    kara.q4_attention(st["p"], st["seqs"], st["case"]["queries"], st["q"], st["kp"], st["vp"], st["ksp"], st["vsp"],
                      st["bt"], st["lens"], st["max_len"], st["out"], st["ws"])
    return dict(out=st["out"])


def _own_weigh(st):
    from paper_2607_01237_amd import kara
    kara.evict_attention(st["p"], st["seqs"], st["q"], st["kp"], st["vp"], st["wp"], st["bt"], st["lens"], 1,
                         st["max_len"], st["out"], st["ws"], k_scales=st["ksp"], v_scales=st["vsp"])
    return dict(out=st["out"], weights=st["weights"][:, :st["pages"]])


def _own_observe(st):
    from paper_2607_01237_amd import kara
    T = st["case"]["queries"]
    kara.evict_observe(st["p"], st["seqs"], T, st["q"], st["kp"], st["wp"], st["bt"], st["lens"], T, st["max_len"],
                       st["ws"], k_scales=st["ksp"])
    return dict(weights=st["weights"][:, :st["pages"]])


def _own_evict(st):
    from paper_2607_01237_amd import kara
    c = st["case"]
    kara.evict_tokens(st["p"], st["seqs"], c["keep"], c["sink"], c["recent"], st["kp"], st["vp"], st["wp"], st["bt"],
                      st["lens"], st["max_len"], True, st["status"], st["ws"], kept=st["kept"], freed=st["freed"],
                      n_freed=st["n_freed"], k_scales=st["ksp"], v_scales=st["vsp"])
    if c["cache"] == "q4":
        kara.q4_read(st["p"], st["seqs"], st["start"], c["keep"], st["kp"], st["vp"], st["ksp"], st["vsp"], st["bt"],
                     st["lens"], st["k_out"], st["v_out"])
    return _evicted(st)


def _evicted(st):
    c = st["case"]
    if c["cache"] == "q4":
        k, v = st["k_out"], st["v_out"]
    else:   # (rows are moved as the bits they hold)
        k, v = (st[x][:, :st["pages"]].view(torch.int32 if c["dtype"] == "f32" else torch.int16) for x in ("k", "v"))
    return dict(kept=st["kept"], freed=st["freed"], n_freed=st["n_freed"], tables=st["bt"], lens=st["lens"],
                status=st["status"], weights=st["weights"][:, :st["pages"]], k=k, v=v)


_own = dict(append=_own_append, attention=_own_attention, weigh=_own_weigh, observe=_own_observe, evict=_own_evict)


# ---- the plain forms

_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _quantize(x):
    """Codes [..., d/2] and scale bytes [..., d/32] of rows [..., d]."""
    b = x.float().unflatten(-1, (-1, 32))
    mag = b.abs()
    top = mag.amax(-1)
    e = (((top.view(torch.int32) + 0x1fffff) >> 23) - 129).clamp_(-125, 125)
    y = torch.ldexp(mag, -e[..., None])
    code = ((y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0)
            + (b < 0).byte() * 8).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).byte()


def _dequantize(codes, scales):
    lut = torch.tensor(_E2M1, device=codes.device)
    x = torch.stack([lut[(codes & 15).long()], lut[(codes >> 4).long()]], dim=-1).flatten(-2)
    s = (scales.to(torch.int32) << 23).view(torch.float32)
    return (x.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _place(st, pos, valid):
    """Pool rows [S][Hkv][positions] of positions pos ([S][positions]); the spare page where not valid."""
    c = st["case"]
    bs, H = c["block"], c["n_kv"]
    table = st["bt"][st["seqs"].long()].long()
    block = pos // bs
    page = torch.where(valid, torch.gather(table, 1, block.clamp(0, table.shape[1] - 1)), st["pages"])
    h = torch.arange(H, device=_DEV)[None, :, None]
    return (page[:, None] * H + h) * bs + (pos % bs)[:, None]


def _flat(pool):
    return pool.view(pool.shape[0], -1, *pool.shape[4:])


def _values(st, which, rows):
    """fp32 rows [L][S][Hkv][positions][d] of the cache."""
    x = _flat(st[which])[:, rows]
    return _dequantize(x, _flat(st[which + "s"])[:, rows]) if which + "s" in st else x.float()


def _plain_append(st):
    c = st["case"]
    lens = st["lens"][st["seqs"].long()].long()
    pos = lens[:, None] + torch.arange(c["new"], device=_DEV)
    rows = _place(st, pos, torch.ones_like(pos, dtype=torch.bool))
    for which in ("k", "v"):
        codes, scales = _quantize(st[which + "_new"].transpose(2, 3))
        _flat(st[which])[:, rows] = codes
        _flat(st[which + "s"])[:, rows] = scales
        st[which + "_out"].copy_(_values(st, which, rows).transpose(2, 3))
    st["lens"][st["seqs"].long()] += c["new"]
    st["status"].zero_()
    return dict(k=st["k_out"], v=st["v_out"], lens=st["lens"], status=st["status"])


def _softmax(st):
    """Unnormalised weights [L][S][Hkv][T * G][positions], their sums, the positions' rows and which are there."""
    c = st["case"]
    L, S, H, G, d, T = c["layers"], c["seqs"], c["n_kv"], c["n_q"] // c["n_kv"], c["d"], c["queries"]
    lens = st["lens"][st["seqs"].long()].long()
    pos = torch.arange(st["max_len"], device=_DEV).expand(S, -1)
    valid = pos < lens[:, None]
    rows = _place(st, pos, valid)
    q = st["q"].float().view(L, S, T, H, G, d).permute(0, 1, 3, 2, 4, 5).reshape(L, S, H, T * G, d)
    k = _values(st, "k", rows)
    s = torch.matmul(q, k.transpose(-1, -2)) * st["scale"]
    last = (lens[:, None] - T + torch.arange(T, device=_DEV)).repeat_interleave(G, dim=1)
    s.masked_fill_((pos[:, None, :] > last[:, :, None])[None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    total = e.sum(-1, keepdim=True)
    return e, torch.where(total == 0, 1.0, total), rows, pos, valid, lens


def _plain_attention(st):
    c = st["case"]
    e, total, rows, _, _, _ = _softmax(st)
    o = torch.matmul(e, _values(st, "v", rows)) / total
    L, S, H, T, G, d = c["layers"], c["seqs"], c["n_kv"], c["queries"], c["n_q"] // c["n_kv"], c["d"]
    st["out"].copy_(o.view(L, S, H, T, G, d).permute(0, 1, 3, 2, 4, 5).reshape(st["out"].shape))
    return dict(out=st["out"])


def _accumulate(st, e, total, rows, pos, valid, lens, n_new):
    w = (e / total).sum(-2)
    flat = _flat(st["weights"])
    fresh = (pos >= lens[:, None] - n_new)[None, :, None]
    flat[:, rows] = torch.where(fresh, 0.0, flat[:, rows]) + w
    return st["weights"][:, :st["pages"]]


def _plain_weigh(st):
    c = st["case"]
    soft = _softmax(st)
    o = torch.matmul(soft[0], _values(st, "v", soft[2])) / soft[1]
    st["out"].copy_(o.reshape(c["layers"], c["seqs"], 1, c["n_q"], c["d"]))
    return dict(out=st["out"], weights=_accumulate(st, *soft, 1))


def _plain_observe(st):
    return dict(weights=_accumulate(st, *_softmax(st), st["case"]["queries"]))


def _plain_evict(st):
    c = st["case"]
    keep, bs = c["keep"], c["block"]
    seqs = st["seqs"].long()
    lens = st["lens"][seqs].long()
    M = max(st["max_len"], keep)
    pos = torch.arange(M, device=_DEV).expand(c["seqs"], -1)
    valid = pos < lens[:, None]
    rows = _place(st, pos, valid)
    w = _flat(st["weights"])[:, rows]
    always = ((pos < c["sink"]) | (pos >= lens[:, None] - c["recent"])) & valid
    w = torch.where(always[None, :, None], math.inf, torch.where(valid[None, :, None], w, -math.inf))
    kept = torch.sort(torch.sort(w, dim=-1, descending=True, stable=True)[1][..., :keep], dim=-1)[0]
    cut = lens > keep
    st["kept"].copy_(torch.where(kept < lens[None, :, None, None], kept, -1))
    src = torch.gather(rows.expand(kept.shape[0], -1, -1, -1), 3, kept)
    dst = torch.where(cut[:, None, None], rows[:, :, :keep], st["pages"] * c["n_kv"] * bs).expand_as(src)
    for x in ("k", "v", "ks", "vs", "weights"):
        if x in st:
            flat = _flat(st[x])
            layer = torch.arange(c["layers"], device=_DEV)[:, None, None, None]
            flat[layer, dst] = flat[layer, src]
    new = torch.where(cut, keep, lens)
    old_b, new_b = (lens + bs - 1) // bs, (new + bs - 1) // bs
    table = st["bt"][seqs].long()
    block = torch.arange(table.shape[1], device=_DEV)
    n = (old_b - new_b)[:, None]
    st["freed"].copy_(torch.where(block < n, torch.gather(table, 1, (block + new_b[:, None]).clamp(max=table.shape[1] - 1)), -1))
    st["n_freed"].copy_(n[:, 0])
    st["bt"][seqs] = torch.where((block >= new_b[:, None]) & (block < old_b[:, None]), -1, table).int()
    st["lens"][seqs] = new.int()
    st["status"].zero_()
    if c["cache"] == "q4":
        at = pos[:, :keep]
        here = at < new[:, None]
        back = _place(st, at, here)
        for x in ("k", "v"):
            st[x + "_out"].copy_((_values(st, x, back) * here[None, :, None, :, None]).transpose(2, 3))
    return _evicted(st)


_plain = dict(append=_plain_append, attention=_plain_attention, weigh=_plain_weigh, observe=_plain_observe,
              evict=_plain_evict)


# ---- from the definitions, in 64 bits

def _grid64(x):
    """The values a cache in 4 bits holds for rows [..., d], fp64."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    mant, ex = torch.frexp(top)                     # top = mant 2^ex, mant in [1/2, 1)
    e = ex - 3 + (mant > 0.875).to(ex.dtype)
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), e.clamp(-125, 125).double())
    y = b.abs() / unit
    even, odd = (torch.tensor(v, dtype=torch.float64, device=x.device) for v in ([0.0, 1.0, 2.0, 4.0], [0.5, 1.5, 3.0, 6.0]))
    pick = lambda grid: (y[..., None] - grid).abs().min(-1)  # noqa: E731
    de, do = pick(even), pick(odd)
    return (torch.where(de[0] <= do[0], even[de[1]], odd[do[1]]) * torch.sign(b) * unit).flatten(-2)


def _cached64(st, which, layer, s, n):
    """Rows [n][Hkv][d] of sequence s in one layer, fp64."""
    bs = st["case"]["block"]
    at = np.arange(n)
    pages = st["bt0"][s].long()[_dev(at // bs)]
    x = st[which][layer][pages, :, _dev(at % bs)]
    if which + "s" not in st:
        return x.double()
    byte = st[which + "s"][layer][pages, :, _dev(at % bs)].double()
    lut = torch.tensor(_E2M1, dtype=torch.float64, device=_DEV)
    out = torch.empty(x.shape[:2] + (2 * x.shape[2],), dtype=torch.float64, device=_DEV)
    out[..., 0::2], out[..., 1::2] = lut[(x % 16).long()], lut[(x // 16).long()]
    return out * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=_DEV), byte - 127).repeat_interleave(32, dim=-1)


def exact(c, seed):
    st = prepare(c, seed)
    L, S, H, G, d = c["layers"], c["seqs"], c["n_kv"], c["n_q"] // c["n_kv"], c["d"]
    if c["kind"] == "append":
        if st["k_new"].numel() > 3e8:
            return None
        k, v = (torch.stack([_grid64(x) for x in st[n].flatten(0, 1)]).view(st[n].shape) for n in ("k_new", "v_new"))
        return dict(k=k, v=v, lens=None, status=None)
    lens, seqs = st["lens0"].tolist(), st["seqs"].tolist()
    if c["kind"] == "evict":
        pool = st["weights0"][:, :st["pages"]].double().cpu().numpy()
        table, bs = st["bt0"].cpu().numpy(), c["block"]
        if L * S * H * c["len_hi"] > 4e7:
            return None
        for layer in range(L):
            for s in seqs:
                n = lens[s]
                if n <= c["keep"]:
                    continue
                at = np.arange(n)
                page, slot = table[s][at // bs], at % bs
                for h in range(H):
                    w = pool[layer, page, h, slot].copy()
                    mid = np.arange(c["sink"], n - c["recent"])
                    best = mid[np.lexsort((mid, -w[mid]))][:c["keep"] - c["sink"] - c["recent"]]
                    kept = np.sort(np.concatenate([at[:c["sink"]], best, at[n - c["recent"]:]]))
                    pool[layer, page[:c["keep"]], h, slot[:c["keep"]]] = w[kept]
        none = dict.fromkeys(("kept", "freed", "n_freed", "tables", "lens", "status", "k", "v"))
        return dict(none, weights=torch.from_numpy(pool))
    T = c["queries"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=_DEV)
    weights = st["weights0"].double() if "weights0" in st else None
    for layer in range(L):
        for j, s in enumerate(seqs):
            n = lens[s]
            k = _cached64(st, "k", layer, s, n).permute(1, 2, 0).contiguous()                          # [H][d][n]
            q = st["q"][layer, j].double().view(T, H, G, d).permute(1, 0, 2, 3).reshape(H, T * G, d)
            x = torch.matmul(q, k) * st["scale"]
            sees = torch.arange(n, device=_DEV) <= (n - T + torch.arange(T, device=_DEV))[:, None]
            hidden = ~sees.repeat_interleave(G, dim=0)
            x = torch.softmax(x.masked_fill(hidden, -math.inf), dim=-1).masked_fill(hidden, 0.0)
            if c["kind"] != "observe":
                v = _cached64(st, "v", layer, s, n).permute(1, 0, 2).contiguous()
                out[layer, j] = torch.matmul(x, v).view(H, T, G, d).permute(1, 0, 2, 3).reshape(T, c["n_q"], d)
            if weights is not None:
                at = torch.arange(n, device=_DEV)
                pages, slot = st["bt0"][s].long()[at // c["block"]], at % c["block"]
                n_new = 1 if c["kind"] == "weigh" else T
                old = weights[layer][pages, :, slot].masked_fill((at >= n - n_new)[:, None], 0.0)
                weights[layer][pages, :, slot] = old + x.sum(1).t()
    res = {}
    if c["kind"] != "observe":
        res["out"] = out
    if weights is not None:
        res["weights"] = weights[:, :st["pages"]]
    return res
