"""Limits of the operators of include/kara_q4.h and include/kara_evict.h, without a GPU."""
import ctypes

import pytest

from paper_2607_01237_amd import kara
from test_abi_operators import CALLS, FAKE, INVALID, UNSUPPORTED, call, lib, params  # noqa: F401


def test_most_tokens_that_a_cut_keeps(lib):  # noqa: F811
    # past 2^31 - 512 the loop that writes a short sequence's positions ran out of its int
    out = ctypes.c_size_t(0)
    for keep in (2 ** 30 + 1, 2 ** 31 - 511, 2 ** 31 - 1):
        assert lib.kara_evict_workspace_size(ctypes.byref(params()), 1, 1, keep, ctypes.byref(out)) == UNSUPPORTED
        assert call(lib, "kara_evict_tokens", keep=keep) == UNSUPPORTED
    assert kara.evict_workspace_size(params(), 1, 1, 2 ** 30) >= 8 * 4 * 2 ** 30


WIDE = {"k_new", "v_new", "q", "k_out", "v_out", "out", "workspace"}


def pools_at(address):
    a = (ctypes.c_void_p * 2)(FAKE, address)
    return a, ctypes.addressof(a)


@pytest.mark.parametrize("name", sorted(CALLS))
def test_unaligned_arrays_are_refused(lib, name):  # noqa: F811
    scales = pools_at(FAKE + 4), pools_at(FAKE + 2)      # of rows of 128: 4 bytes each
    change = {}
    if "k_scales" in dict(CALLS[name]):
        change = {x: scales[0][1] for x in ("k_scales", "v_scales") if x in dict(CALLS[name])}
    for key, good in CALLS[name]:
        if key in WIDE:
            assert call(lib, name, **{key: FAKE + 8}, **change) == INVALID, key
        elif good == FAKE or key == "kept":
            assert call(lib, name, **{key: FAKE + 2}, **change) == INVALID, key
        elif key in ("k_pools", "v_pools", "weights"):
            held, at = pools_at(FAKE + 8)
            assert call(lib, name, **{key: at}, **change) == INVALID, key
        elif key.endswith("_scales"):
            assert call(lib, name, **dict(change, **{key: scales[1][1]})) == INVALID, key
    if "weights" in dict(CALLS[name]):                   # pages of three tokens: accumulators one at a time
        held, at = pools_at(FAKE + 2)
        assert call(lib, name, params(block_size=3, max_blocks_per_seq=400), weights=at) == INVALID


def test_binding_refuses_missing_accumulators():
    torch = pytest.importorskip("torch")
    x = [torch.zeros(8 * 16 * 128, dtype=torch.bfloat16)]
    for values in (True, False):
        with pytest.raises(kara.KaraError, match="weights: missing"):
            kara._cache_args(torch, -1, params(num_pages=1), 1, x, x, None, None, None, values=values)
    assert len(kara._cache_args(torch, -1, params(num_pages=1), 1, x, x, None, None)[1]) == 4


def test_binding_takes_layers_of_one_tensor():
    torch = pytest.importorskip("torch")
    rows, w = torch.zeros((2, 8 * 16 * 128), dtype=torch.bfloat16), torch.zeros((2, 8 * 16))
    held, at = kara._cache_args(torch, -1, params(num_pages=1), 2, rows, rows, None, None, w)
    assert list(held) == [t.data_ptr() for x in (rows, rows, w) for t in x]


def test_workspace_sizes_the_headers_name(lib):  # noqa: F811
    # one for each n_query: a decoding step over many sequences needs more than a chunk of a prompt
    p = params(max_blocks_per_seq=2000)
    step, chunk = (kara.q4_attention_workspace_size(p, 100, 1, t, 32000) for t in (1, 300))
    assert step == 100 * 32 * 125 * 130 * 4 and 33e6 < chunk < 35e6
    args = dict(n=8, n_layers=1, max_len=32000)
    small = kara.q4_attention_workspace_size(p, 8, 1, 300, 32000) // 4
    assert call(lib, "kara_q4_attention", p, n_query=1, bytes=small, **args) == kara.ERR_WORKSPACE
    few = params(max_blocks_per_seq=2048, n_q_heads=40)
    assert 0.50e9 < kara.evict_attention_workspace_size(few, 64, 1, 32768) < 0.51e9
