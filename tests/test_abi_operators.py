"""The operators of include/kara_q4.h and include/kara_evict.h without a GPU: every
declared function is exported and bound, and bad calls are refused before
anything is launched."""
import ctypes
import itertools
import os

import pytest

from paper_2607_01237_amd import kara

FAKE = 0x1000            # never dereferenced
INVALID, UNSUPPORTED, WORKSPACE, OK = kara.ERR_INVALID_ARG, kara.ERR_UNSUPPORTED, kara.ERR_WORKSPACE, kara.OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kara.LIB_PATH):
        from paper_2607_01237_amd import build
        build.build()
    return kara.load()


def params(**kw):
    p = dict(window=64, buffer=0, budget=16, chunk_budget=4, max_chunk_len=4, head_dim=128, n_q_heads=32, n_kv_heads=8,
             block_size=16, num_pages=4096, max_blocks_per_seq=200, dtype="bf16", scale=0.0)
    p.update(kw)
    return kara.make_params(p, n_seqs=8)


_pools = (ctypes.c_void_p * 80)(*([FAKE] * 80))
POOLS = ctypes.addressof(_pools)
_holes = (ctypes.c_void_p * 2)(FAKE, None)
HOLES = ctypes.addressof(_holes)
BIG = 1 << 40

# name: (arguments after p, in order, each a (key, good value))
CALLS = {
    "kara_q4_append": [("n", 2), ("seqs", FAKE), ("n_new", 3), ("n_layers", 2), ("k_new", FAKE), ("v_new", FAKE),
                       ("k_pools", POOLS), ("v_pools", POOLS), ("k_scales", POOLS), ("v_scales", POOLS),
                       ("block_table", FAKE), ("seq_lens", FAKE), ("status", FAKE), ("stream", None)],
    "kara_q4_read": [("n", 2), ("seqs", FAKE), ("start", FAKE), ("n_rows", 3), ("n_layers", 2), ("k_pools", POOLS),
                     ("v_pools", POOLS), ("k_scales", POOLS), ("v_scales", POOLS), ("block_table", FAKE),
                     ("seq_lens", FAKE), ("k_out", FAKE), ("v_out", FAKE), ("stream", None)],
    "kara_q4_attention": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("n_query", 3), ("q", FAKE), ("k_pools", POOLS),
                          ("v_pools", POOLS), ("k_scales", POOLS), ("v_scales", POOLS), ("block_table", FAKE),
                          ("seq_lens", FAKE), ("max_len", 1000), ("out", FAKE), ("workspace", FAKE), ("bytes", BIG),
                          ("stream", None)],
    "kara_evict_attention": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("q", FAKE), ("k_pools", POOLS),
                             ("v_pools", POOLS), ("k_scales", None), ("v_scales", None), ("weights", POOLS),
                             ("block_table", FAKE), ("seq_lens", FAKE), ("n_new", 1), ("max_len", 1000), ("out", FAKE),
                             ("workspace", FAKE), ("bytes", BIG), ("stream", None)],
    "kara_evict_observe": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("n_query", 3), ("q", FAKE), ("k_pools", POOLS),
                           ("k_scales", None), ("weights", POOLS), ("block_table", FAKE), ("seq_lens", FAKE),
                           ("n_new", 3), ("max_len", 1000), ("workspace", FAKE), ("bytes", BIG), ("stream", None)],
    "kara_evict_tokens": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("keep", 100), ("n_sink", 4), ("n_recent", 10),
                          ("k_pools", POOLS), ("v_pools", POOLS), ("k_scales", None), ("v_scales", None),
                          ("weights", POOLS), ("block_table", FAKE), ("seq_lens", FAKE), ("max_len", 1000), ("commit", 1),
                          ("kept", None), ("freed", FAKE), ("n_freed", FAKE), ("status", FAKE), ("workspace", FAKE),
                          ("bytes", BIG), ("stream", None)],
}
OPTIONAL = {"stream", "kept", "k_scales", "v_scales"}


def call(lib, name, p=None, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    return getattr(lib, name)(ctypes.byref(p or params()), *args.values())


def test_exports_and_binds_every_declared_function(lib):
    names = kara.header_functions(kara.OPERATOR_HEADERS)
    assert len(names) == 10, names
    for n in names:
        assert hasattr(lib, n) and n in kara._SIGS, n
    assert set(CALLS) == {n for n in names if not n.endswith("workspace_size")}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(lib, name):
    args = dict(CALLS[name])
    # nothing listed is no error and touches no pointer
    assert call(lib, name, n=0) == OK
    if "n_new" in args and name == "kara_q4_append":
        assert call(lib, name, n_new=0) == OK
    if "n_rows" in args:
        assert call(lib, name, n_rows=0) == OK
    for key, good in args.items():
        if good in (FAKE, POOLS) and key != "workspace":
            assert call(lib, name, **{key: None}) == INVALID, key
        if good == POOLS:
            assert call(lib, name, **{key: HOLES}) == INVALID, key
        if key in ("n", "n_new", "n_rows", "n_sink", "n_recent"):
            assert call(lib, name, **{key: -1}) == INVALID, key
        if key in ("n_query", "keep", "max_len", "n_layers"):
            assert call(lib, name, **{key: 0}) == INVALID, key
        if key == "max_len":                              # past what the table maps
            assert call(lib, name, max_len=200 * 16 + 1) == INVALID
    assert call(lib, name, n_layers=65) == INVALID
    assert getattr(lib, name)(None, *args.values()) == INVALID
    for bad, code in ((dict(head_dim=96), UNSUPPORTED), (dict(n_q_heads=30), INVALID), (dict(block_size=0), INVALID),
                      (dict(dtype=7), INVALID), (dict(num_pages=1 << 30), UNSUPPORTED)):
        assert call(lib, name, params(**bad)) == code, bad
    if "workspace" in args:
        assert call(lib, name, workspace=None) == WORKSPACE
        assert call(lib, name, bytes=4) == WORKSPACE


def test_refusals_of_their_own(lib):
    for name in ("kara_evict_attention", "kara_evict_tokens"):         # both scale arrays or neither
        assert call(lib, name, k_scales=POOLS) == INVALID
        assert call(lib, name, v_scales=POOLS) == INVALID
        assert call(lib, name, k_scales=POOLS, v_scales=HOLES) == INVALID
    assert call(lib, "kara_evict_observe", k_scales=HOLES) == INVALID
    assert call(lib, "kara_evict_attention", params(n_q_heads=136)) == UNSUPPORTED       # 17 heads in a group
    assert call(lib, "kara_evict_tokens", n_sink=91) == INVALID                          # 91 + 10 > 100
    assert call(lib, "kara_evict_tokens", n_sink=2**31 - 1, n_recent=2**31 - 1) == INVALID
    assert call(lib, "kara_evict_tokens", freed=None) == INVALID
    assert call(lib, "kara_evict_tokens", kept=FAKE, bytes=7) == WORKSPACE               # the lengths alone: 8 bytes
    # grids past what one launch holds
    assert call(lib, "kara_q4_append", n_new=2**30, n=64) == UNSUPPORTED
    assert call(lib, "kara_evict_tokens", n=2**20) == UNSUPPORTED


def test_workspaces_cover_smaller_launches(lib):
    # a server sizes a workspace once: what fewer sequences, layers or a shorter
    # longest sequence need must fit it
    p = params(max_blocks_per_seq=2000)
    counts = [1, 2, 3, 5, 8, 15, 16, 17, 31, 64, 100]
    for size in (lambda n, layers, m: kara.q4_attention_workspace_size(p, n, layers, 1, m),
                 lambda n, layers, m: kara.q4_attention_workspace_size(p, n, layers, 7, m),
                 lambda n, layers, m: kara.q4_attention_workspace_size(p, n, layers, 300, m),
                 lambda n, layers, m: kara.evict_attention_workspace_size(p, n, layers, m),
                 lambda n, layers, m: kara.evict_observe_workspace_size(p, n, layers, 50, m),
                 lambda n, layers, m: kara.evict_workspace_size(p, n, layers, m)):
        for layers, m in itertools.product((1, 3, 64), (1, 255, 257, 5000, 32000)):
            sizes = [size(n, layers, m) for n in counts]
            assert all(a <= b for a, b in zip(sizes, sizes[1:]))
        for n in counts:
            sizes = [size(n, 3, m) for m in (1, 255, 256, 257, 511, 5000, 32000)]
            assert all(a <= b for a, b in zip(sizes, sizes[1:]))
            assert size(n, 1, 5000) <= size(n, 2, 5000)
    out = ctypes.c_size_t(0)
    for name in ("kara_q4_attention", "kara_evict_observe"):
        assert getattr(lib, name + "_workspace_size")(ctypes.byref(p), 2, 1, 1, 100, None) == INVALID
        assert getattr(lib, name + "_workspace_size")(ctypes.byref(p), 2, 1, 2**30, 100, ctypes.byref(out)) == INVALID


def test_binding_checks():
    torch = pytest.importorskip("torch")
    cpu = -1                                              # the device index of a CPU tensor
    x = torch.zeros((4, 6), dtype=torch.float32)
    assert kara._arg(cpu, "x", x, 24, torch.float32) == x.data_ptr()
    for bad, what in ((dict(n=25), "at least 25"), (dict(dtype=torch.int32), "dtype"), (dict(t=None), "missing"),
                      (dict(t=x.t()), "contiguous"), (dict(dev=0), "current device")):
        a = dict(dev=cpu, name="x", t=x, n=24, dtype=torch.float32, **{})
        a.update(bad)
        with pytest.raises(kara.KaraError, match=what):
            kara._arg(a["dev"], a["name"], a["t"], a["n"], a["dtype"])
    p = params(num_pages=3)
    rows = 3 * 8 * 16
    codes = [torch.zeros(rows * 64, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros(rows * 4, dtype=torch.uint8) for _ in range(2)]
    weights = [torch.zeros(rows) for _ in range(2)]
    held, at = kara._cache_args(torch, cpu, p, 2, codes, codes, scales, scales, weights)
    assert len(held) == 10 and [a is None for a in at] == [False] * 5
    assert [ctypes.c_void_p.from_address(at[2] + 8 * i).value for i in range(2)] == [t.data_ptr() for t in scales]
    rows16 = [torch.zeros(rows * 128, dtype=torch.bfloat16) for _ in range(2)]
    held, at = kara._cache_args(torch, cpu, p, 2, rows16, rows16, None, None, weights)
    assert len(held) == 6 and at[2] is None and at[3] is None
    for bad in ((codes, codes, None, None, weights), (codes, codes, scales, None, weights),
                (codes, codes[:1], scales, scales, weights), (codes, codes, scales, scales, [None, weights[0]]),
                (codes, codes, [scales[0][1:], scales[1]], scales, weights)):
        with pytest.raises(kara.KaraError):
            kara._cache_args(torch, cpu, p, 2, *bad)


def test_longest_sequences(lib):
    # max_len up to 2^30, whatever the table could map; sizes there do not wrap
    out = ctypes.c_size_t(0)
    p = params(block_size=256, num_pages=1, max_blocks_per_seq=(2 ** 31 - 1) // 256)
    sizes = {"kara_q4_attention_workspace_size": (1, 1, 1), "kara_evict_attention_workspace_size": (1, 1),
             "kara_evict_observe_workspace_size": (1, 1, 4)}
    for name, args in sizes.items():
        fn = getattr(lib, name)
        assert fn(ctypes.byref(p), *args, 2 ** 30, ctypes.byref(out)) == OK
        if "observe" not in name:                      # a record per 256 keys and query head
            assert out.value >= 2 ** 22 * 32 * 130 * 4, name
        assert fn(ctypes.byref(p), *args, 2 ** 30 + 1, ctypes.byref(out)) == UNSUPPORTED, name
    for name in ("kara_q4_attention", "kara_evict_attention", "kara_evict_observe", "kara_evict_tokens"):
        args = [2 ** 30 + 1 if k == "max_len" else v for k, v in CALLS[name]]
        assert getattr(lib, name)(ctypes.byref(p), *args) == UNSUPPORTED, name
