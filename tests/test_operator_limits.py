"""Limits of the operators of include/kara_q4.h and include/kara_evict.h, without a GPU."""
import ctypes

from paper_2607_01237_amd import kara
from test_abi_operators import UNSUPPORTED, call, lib, params  # noqa: F401


def test_most_tokens_that_a_cut_keeps(lib):  # noqa: F811
    # past 2^31 - 512 the loop that writes a short sequence's positions ran out of its int
    out = ctypes.c_size_t(0)
    for keep in (2 ** 30 + 1, 2 ** 31 - 511, 2 ** 31 - 1):
        assert lib.kara_evict_workspace_size(ctypes.byref(params()), 1, 1, keep, ctypes.byref(out)) == UNSUPPORTED
        assert call(lib, "kara_evict_tokens", keep=keep) == UNSUPPORTED
    assert kara.evict_workspace_size(params(), 1, 1, 2 ** 30) >= 8 * 4 * 2 ** 30
