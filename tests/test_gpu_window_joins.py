"""Windowed attention (include/kara_window.h) gives what its formula gives however keys are
split: parts of a sequence whose every logit is -inf, and the values they hold."""
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


NAN_COLUMN, INF_COLUMN, N, DEAD = 5, 40, 4000, 2000


def _call(layers, T, dtype, k, v, q, table, lens):
    from paper_2607_01237_amd import kara
    pages, Hkv, bs, d = k.shape
    Hq = q.shape[1]
    p = cc.params(Hq, Hkv, d, bs, pages, table.shape[1], len(lens), dtype)
    seqs = cc.gpu(np.arange(len(lens), dtype=np.int32))
    qs = q.expand(layers, len(lens), *q.shape).contiguous()
    out = torch.full_like(qs, 7.0)
    need = kara.window_attention_workspace_size(p, len(lens), layers, T, 0, 0, N)
    ws = torch.full((max(1, need),), 255, dtype=torch.uint8, device="cuda")
    kara.window_attention(p, seqs, T, 0, 0, qs, [k] * layers, [v] * layers, cc.gpu(table), cc.gpu(lens), N, out, ws)
    return out


@pytest.mark.parametrize("dead", ["first", "last", "all"])
@pytest.mark.parametrize("dtype,d,T", [("bf16", 64, 1), ("bf16", 128, 5), ("bf16", 64, 120), ("bf16", 128, 300), ("f32", 64, 1),
                                       ("f32", 128, 40)])
def test_values_of_logits_of_minus_infinity_enter_however_keys_are_split(dtype, d, T, dead):
    # Half of a sequence's keys have logits of -inf: its other keys alone have weight, but what
    # is not finite among the values it sees enters, as 0 times an infinity or a NaN does.  One
    # layer's keys are split; 64 layers of 8 KV heads fill the card, and are not.
    rng = np.random.default_rng(d + T)
    Hq, Hkv, bs = 16, 8, 16
    lens = np.array([N], dtype=np.int32)
    table, pages, _ = cc.table_for(rng, lens, bs, N // bs)
    k, v = (torch.from_numpy(rng.standard_normal((pages, Hkv, bs, d)).astype(np.float32)).to(cc.DT[dtype]).cuda() for _ in range(2))
    at = np.arange(N)
    gone = dict(first=at < DEAD, last=at >= DEAD, all=at >= 0)[dead]
    page, slot = torch.from_numpy(table[0][at // bs]).long().cuda(), torch.from_numpy(at % bs).cuda()
    is_gone = torch.from_numpy(gone).cuda()
    k[page[is_gone], :, slot[is_gone], 0] = float("-inf")
    for pos in np.flatnonzero(gone[:N - T])[[900, 1500]]:          # (every query sees them)
        v[page[pos], :, slot[pos], NAN_COLUMN] = float("nan")
        v[page[pos], :, slot[pos], INF_COLUMN] = float("inf")
    q = torch.from_numpy(rng.standard_normal((T, Hq, d)).astype(np.float32)).abs().to(cc.DT[dtype]).cuda()
    split, whole = (_call(layers, T, dtype, k, v, q, table, lens) for layers in (1, 64))
    k64, v64 = (t[page, :, slot].double().cpu().numpy() for t in (k, v))
    for name, out in (("split", split[0, 0]), ("whole", whole[0, 0]), ("whole, last layer", whole[63, 0])):
        got = out.double().cpu().numpy()
        if dead == "all":                                          # no weight at all: zero, whatever the values
            assert not got.any(), name
            continue
        assert np.isnan(got[..., NAN_COLUMN]).all(), name
        assert not np.isfinite(got[..., INF_COLUMN]).any(), name
        for t in {0, T // 2, T - 1}:
            n = N - T + t + 1
            ref, mass = ks.attend(q[t:t + 1].double().cpu().numpy(), k64[:n], v64[:n], 1 / np.sqrt(d))
            sane = np.where(np.isfinite(k64), k64, 0.0)
            delta = cc.logit_error(q[t:t + 1].double().cpu().numpy(), sane[:n], 1 / np.sqrt(d), 1 if dtype == "bf16" else 3)
            bound = cc.attention_bound(ref, mass, delta, n, dtype, dtype == "bf16")
            fine = np.ones(d, bool)
            fine[[NAN_COLUMN, INF_COLUMN]] = False
            assert (np.abs(got[t] - ref[0]) <= bound[0])[:, fine].all(), (name, t)
            assert np.isnan(ref[..., NAN_COLUMN]).all() and not np.isfinite(ref[..., INF_COLUMN]).any()
