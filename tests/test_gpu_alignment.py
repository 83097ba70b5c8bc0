"""Caches whose layers lie in one tensor, pages of an odd number of tokens: scales on
2 bytes and accumulators on 4, the least that include/kara_evict.h asks for."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

import cache_check as cc  # noqa: E402
from test_gpu_evict import Cache, check_evict, count_case, observe_case, run_evict  # noqa: E402
from test_gpu_q4 import _kara  # noqa: E402


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


LENS = [1, 31, 0, 256, 257, 600, 90]                    # (seven more each: 186 pages of 7, and five)


@pytest.mark.parametrize("kind", ["q4", "rows"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_least_alignment(kind, dtype):
    print(f"\n[case] alignment {kind} {dtype}", flush=True)
    lens, seqs = [n + 7 for n in LENS], list(range(7))
    c = Cache(np.random.default_rng(4), kind, dtype, 3, 1, 64, 7, lens, layers=3)
    assert c.pages % 2 == 1 and c.weights[1].data_ptr() % 16 != 0
    if kind == "q4":
        assert c.dev["ks"][1].data_ptr() % 4 == 2
    shape = (kind, dtype, 3, 1, 64, 7, 3)
    assert max(count_case(*shape, 1, lens, max(lens), seqs)) < 1
    for T in (2, 150):
        assert observe_case(*shape, T, 1, lens, max(lens), seqs) < 1
    check_evict(c, seqs, {}, 100, 2, 30, run_evict(c, seqs, 100, 2, 30, max(lens)))


def test_least_alignment_of_a_4_bit_cache():
    kara = _kara()
    c = Cache(np.random.default_rng(5), "q4", "bf16", 3, 1, 64, 7, [n + 7 for n in LENS], layers=3)
    lists = c.lists("k", "v", "ks", "vs")
    aligned = [[t.clone() for t in x] for x in lists]
    store = torch.zeros(8, dtype=torch.int32, device="cuda")
    seqs, status = store[1:], torch.full((9,), 9, dtype=torch.int32, device="cuda")[2:]
    seqs.copy_(torch.arange(7, dtype=torch.int32))
    start = cc.gpu(np.zeros(7, dtype=np.int32))
    for n_new, T in ((1, 1), (7, 5), (7, 60)):
        x = torch.randn((2, 3, 7, n_new, 1, 64), device="cuda").bfloat16()
        q = torch.randn((3, 7, T, 3, 64), device="cuda").bfloat16()
        got = []
        for pools in (lists, aligned):
            sl = cc.gpu(np.maximum(c.lens - n_new, 0))
            kara.q4_append(c.p, seqs, x[0], x[1], *pools, c.bt, sl, status)
            out, k, v = torch.empty_like(q), *(torch.empty((3, 7, 600, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            ws = torch.empty(kara.q4_attention_workspace_size(c.p, 7, 3, T, 607), dtype=torch.uint8, device="cuda")
            kara.q4_attention(c.p, seqs, T, q, *pools, c.bt, sl, 607, out, ws)
            kara.q4_read(c.p, seqs, start, 600, *pools, c.bt, sl, k, v)
            assert not status.any()
            got.append([out, k, v, *pools[0], *pools[1], *pools[2], *pools[3]])
        for a, b in zip(*got):
            assert torch.equal(a, b)


def test_unaligned_tensors_are_refused():
    kara = _kara()
    c = Cache(np.random.default_rng(6), "q4", "bf16", 8, 2, 128, 16, [40, 30])
    k, v, ks, vs = c.lists("k", "v", "ks", "vs")

    def off(t, by):
        held = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")
        return held[by:].view(t.shape).copy_(t)

    q = torch.randn((1, 2, 1, 8, 128), device="cuda").bfloat16()
    out = torch.full((1, 2, 1, 8, 128), 3.0, device="cuda")
    ws = torch.empty(kara.evict_attention_workspace_size(c.p, 2, 1, 40), dtype=torch.uint8, device="cuda")
    good = dict(p=c.p, seqs=cc.gpu(np.arange(2, dtype=np.int32)), q=q, k_pools=k, v_pools=v, weights=c.weights,
                block_table=c.bt, seq_lens=c.sl, n_new=1, max_len=40, out=out, workspace=ws, k_scales=ks, v_scales=vs)
    for bad in (dict(q=off(q, 1)), dict(out=off(out, 2)), dict(k_pools=[off(k[0], 8)]), dict(v_scales=[off(vs[0], 2)]),
                dict(weights=[off(c.weights[0], 1)]), dict(workspace=off(ws, 4))):
        with pytest.raises(kara.KaraError, match="not aligned"):
            kara.evict_attention(**dict(good, **bad))
    assert bool((out == 3.0).all())
    kara.evict_attention(**dict(good, k_scales=[off(ks[0], 4)], seqs=off(good["seqs"], 1)))
    assert not bool((out == 3.0).any())
