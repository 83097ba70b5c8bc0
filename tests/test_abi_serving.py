"""The operators of include/kara_q8.h, kara_rope.h and kara_window.h without a GPU: every
declared function is exported and bound, and bad calls are refused before anything is
launched."""
import ctypes
import itertools
import os

import pytest

from paper_2607_01237_amd import kara
from test_abi_operators import BIG, FAKE, HOLES, INVALID, OK, POOLS, UNSUPPORTED, WORKSPACE, params


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kara.LIB_PATH):
        from paper_2607_01237_amd import build
        build.build()
    return kara.load()


_odd = (ctypes.c_void_p * 80)(*([FAKE + 8] * 80))        # pools that are not aligned
ODD = ctypes.addressof(_odd)
ROPE = kara.make_rope(theta=1e6)
_ROPE = ctypes.addressof(ROPE)

# name: (arguments after p, in order, each a (key, good value))
_CACHE = [("k_pools", POOLS), ("v_pools", POOLS), ("k_scales", POOLS), ("v_scales", POOLS), ("block_table", FAKE),
          ("seq_lens", FAKE)]
CALLS = {
    "kara_q8_append": [("n", 2), ("seqs", FAKE), ("n_new", 3), ("n_layers", 2), ("k_new", FAKE), ("v_new", FAKE), *_CACHE,
                       ("status", FAKE), ("stream", None)],
    "kara_q8_read": [("n", 2), ("seqs", FAKE), ("start", FAKE), ("n_rows", 3), ("n_layers", 2), *_CACHE, ("k_out", FAKE),
                     ("v_out", FAKE), ("stream", None)],
    "kara_q8_attention": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("n_query", 3), ("q", FAKE), *_CACHE,
                          ("max_len", 1000), ("out", FAKE), ("workspace", FAKE), ("bytes", BIG), ("stream", None)],
    "kara_rope_append": [("rope", ctypes.cast(_ROPE, ctypes.POINTER(kara.KaraRope))), ("n", 2), ("seqs", FAKE), ("n_new", 3),
                         ("n_layers", 2), ("q", None), ("k_new", FAKE), ("v_new", FAKE), ("q_out", None),
                         ("k_pools", POOLS), ("v_pools", POOLS), ("k_scales", None), ("v_scales", None),
                         ("block_table", FAKE), ("seq_lens", FAKE), ("rope_pos", None), ("counted", 0), ("status", FAKE),
                         ("stream", None)],
    "kara_window_attention": [("n", 2), ("seqs", FAKE), ("n_layers", 2), ("n_query", 3), ("window", 500), ("n_sink", 4),
                              ("q", FAKE), ("k_pools", POOLS), ("v_pools", POOLS), ("k_scales", None), ("v_scales", None),
                              ("block_table", FAKE), ("seq_lens", FAKE), ("max_len", 1000), ("out", FAKE),
                              ("workspace", FAKE), ("bytes", BIG), ("stream", None)],
}


def call(lib, name, p=None, **change):
    args = dict(CALLS[name])
    assert set(change) <= set(args)
    args.update(change)
    return getattr(lib, name)(ctypes.byref(p or params()), *args.values())


def test_exports_and_binds_every_declared_function(lib):
    names = kara.header_functions(kara.SERVING_HEADERS)
    assert len(names) == 7, names
    for n in names:
        assert hasattr(lib, n) and n in kara._SIGS, n
    assert set(CALLS) == {n for n in names if not n.endswith("workspace_size")}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_refusals(lib, name):
    args = dict(CALLS[name])
    # nothing listed is no error and touches no pointer
    assert call(lib, name, n=0) == OK
    for key in ("n_new", "n_rows"):
        if key in args:
            assert call(lib, name, **{key: 0}) == OK
    for key, good in args.items():
        if key == "workspace":
            continue
        if key == "rope":
            assert call(lib, name, rope=None) == INVALID
        elif good in (FAKE, POOLS):
            assert call(lib, name, **{key: None}) == INVALID, key
        if key != "rope" and good == POOLS:
            assert call(lib, name, **{key: HOLES}) == INVALID, key
            if not key.endswith("scales"):                # (bytes lie anywhere)
                assert call(lib, name, **{key: ODD}) == INVALID, key
        if key != "rope" and good == FAKE:                # alignment
            assert call(lib, name, **{key: FAKE + 2}) == INVALID, key
        if key in ("n", "n_new", "n_rows", "n_sink", "window", "counted"):
            assert call(lib, name, **{key: -1}) == INVALID, key
        if key in ("n_query", "max_len", "n_layers"):
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
    for name in ("kara_rope_append", "kara_window_attention"):         # both scale arrays or neither
        assert call(lib, name, k_scales=POOLS) == INVALID
        assert call(lib, name, v_scales=POOLS) == INVALID
        assert call(lib, name, k_scales=POOLS, v_scales=HOLES) == INVALID
    assert call(lib, "kara_rope_append", q=FAKE) == INVALID             # both queries or neither
    assert call(lib, "kara_rope_append", q_out=FAKE) == INVALID
    assert call(lib, "kara_rope_append", counted=2) == INVALID
    assert call(lib, "kara_rope_append", rope_pos=FAKE + 2) == INVALID
    for bad in (dict(dim=8), dict(dim=144), dict(dim=-16), dict(theta=0.0), dict(theta=-1.0), dict(theta=float("inf")),
                dict(theta=float("nan"))):
        r = kara.make_rope(**bad)
        assert call(lib, "kara_rope_append", rope=ctypes.pointer(r)) == INVALID, bad
    r = kara.KaraRope(0, 1e6, FAKE + 2)
    assert call(lib, "kara_rope_append", rope=ctypes.pointer(r)) == INVALID
    # grids past what one launch holds
    for name in ("kara_q8_append", "kara_rope_append"):
        assert call(lib, name, n_new=2**30, n=64) == UNSUPPORTED
    assert call(lib, "kara_q8_read", n_rows=2**30, n=64) == UNSUPPORTED
    for name in ("kara_q8_append", "kara_rope_append"):                 # heads whose items leave 32 bits
        assert call(lib, name, params(n_q_heads=2**19, n_kv_heads=2**19, num_pages=1)) == UNSUPPORTED


def test_workspaces_cover_smaller_launches(lib):
    # a server sizes a workspace once: what fewer sequences, layers or a shorter
    # longest sequence need must fit it
    counts = [1, 2, 3, 5, 8, 15, 16, 17, 31, 64, 100]
    for dtype, bs in (("bf16", 16), ("f32", 7)):
        p = params(max_blocks_per_seq=32000 // bs + 1, block_size=bs, dtype=dtype)
        sizes = [lambda n, layers, m, T=T: kara.q8_attention_workspace_size(p, n, layers, T, m) for T in (1, 7, 300)]
        sizes += [lambda n, layers, m, T=T, w=w, s=s: kara.window_attention_workspace_size(p, n, layers, T, w, s, m)
                  for T, w, s in itertools.product((1, 7, 300), (0, 1, 500, 20000), (0, 4, 5000))]
        for size in sizes:
            for layers, m in itertools.product((1, 3, 64), (1, 255, 257, 5000, 32000)):
                got = [size(n, layers, m) for n in counts]
                assert all(a <= b for a, b in zip(got, got[1:]))
            for n in counts:
                got = [size(n, 3, m) for m in (1, 255, 256, 257, 511, 5000, 32000)]
                assert all(a <= b for a, b in zip(got, got[1:]))
                assert size(n, 1, 5000) <= size(n, 2, 5000)
    out = ctypes.c_size_t(0)
    p = params(max_blocks_per_seq=2000)
    for name, more in (("kara_q8_attention", ()), ("kara_window_attention", (9, 9))):
        fn = getattr(lib, name + "_workspace_size")
        assert fn(ctypes.byref(p), 2, 1, 1, *more, 100, None) == INVALID
        assert fn(ctypes.byref(p), 2, 1, 2**30, *more, 100, ctypes.byref(out)) == INVALID
        assert fn(ctypes.byref(p), 2, 1, 0, *more, 100, ctypes.byref(out)) == INVALID


def test_longest_sequences(lib):
    # max_len up to 2^30, whatever the table could map; sizes there do not wrap
    out = ctypes.c_size_t(0)
    p = params(block_size=256, num_pages=1, max_blocks_per_seq=(2 ** 31 - 1) // 256)
    for name, args in (("kara_q8_attention", (1, 1, 1)), ("kara_window_attention", (1, 1, 1, 0, 0)),
                       ("kara_window_attention", (1, 1, 1, 2**31 - 1, 2**31 - 1))):
        fn = getattr(lib, name + "_workspace_size")
        assert fn(ctypes.byref(p), *args, 2 ** 30, ctypes.byref(out)) == OK
        assert out.value >= 2 ** 30 // 4608 * 32 * 130 * 4, name       # a record per 4608 keys and query head
        assert fn(ctypes.byref(p), *args, 2 ** 30 + 1, ctypes.byref(out)) == UNSUPPORTED, name
    # in a window the size does not grow with the sequence
    sizes = [kara.window_attention_workspace_size(p, 4, 1, 1, 1000, 4, m) for m in (2000, 2 ** 20, 2 ** 30)]
    assert sizes[0] == sizes[1] == sizes[2]
    for name in ("kara_q8_attention", "kara_window_attention"):
        args = [2 ** 30 + 1 if k == "max_len" else v for k, v in CALLS[name]]
        assert getattr(lib, name)(ctypes.byref(p), *args) == UNSUPPORTED, name


def test_binding_checks():
    torch = pytest.importorskip("torch")
    cpu = -1                                              # the device index of a CPU tensor
    p = params(num_pages=3)
    units = 3 * 8
    codes = [torch.zeros(units * 16 * 128, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.zeros(units, dtype=torch.uint8) for _ in range(2)]
    rows = [torch.zeros(units * 16 * 128, dtype=torch.bfloat16) for _ in range(2)]
    addresses = lambda b: list(memoryview(b).cast("Q"))  # noqa: E731
    at = kara._rows_or_q8_args(torch, cpu, p, 2, codes, codes, scales, scales)
    assert [addresses(b) for b in at] == [[t.data_ptr() for t in ts] for ts in (codes, codes, scales, scales)]
    at = kara._rows_or_q8_args(torch, cpu, p, 1, rows[:1], rows[1:], None, None)
    assert [addresses(b) for b in at[:2]] == [[t.data_ptr()] for t in rows] and at[2] is None and at[3] is None
    assert ctypes.cast(ctypes.c_char_p(at[0]), ctypes.POINTER(ctypes.c_void_p))[0] == rows[0].data_ptr()
    for bad in ((codes, codes, None, None), (rows, rows, scales, scales), (codes, codes, scales, None),
                (codes, codes[:1], scales, scales), (codes, codes, [scales[0][1:], scales[1]], scales)):
        with pytest.raises(kara.KaraError):
            kara._rows_or_q8_args(torch, cpu, p, 2, *bad)
    with pytest.raises(kara.KaraError):
        kara.make_rope(dim=128, inv_freq=torch.zeros(63))
    r = kara.make_rope(dim=64, inv_freq=torch.zeros(32))
    assert r.inv_freq == r.held.data_ptr()
