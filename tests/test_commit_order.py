"""Calls of several launches commit last.  Eviction: tables and lengths reach them read-only,
but for the one that moves the rows, which comes after the others.  (A launch that
fails cannot be had from valid arguments, so the source says it.)"""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_01237_amd", "csrc", "kara_evict.hip")


def test_only_the_last_launch_writes_tables_and_lengths():
    text = open(SRC).read()
    args = re.search(r"struct EvictArgs \{(.*?)\n\};", text, re.S).group(1)
    const = re.search(r"const int32_t ([^;]*);", args).group(1)
    assert {"*bt", "*seq_lens"} <= set(const.split(", "))
    kernels = re.findall(r"void (evict_\w+_kernel)\(([^)]*)\)", text)
    takes = {name: params for name, params in kernels if "EvictArgs" in params}
    assert set(takes) == {"evict_validate_kernel", "evict_pick_kernel", "evict_move_kernel"}
    assert [name for name, params in takes.items() if params != "EvictArgs a"] == ["evict_move_kernel"]
    body = text[text.index("kara_status_t kara_evict_tokens("):]
    launched = re.findall(r"hipLaunchKernelGGL\(\(?(evict_\w+_kernel)", body)
    assert launched == ["evict_validate_kernel", "evict_pick_kernel", "evict_move_kernel", "evict_move_kernel"]
    assert "const_cast<int32_t" not in text


def test_a_long_append_commits_last():
    text = open(os.path.join(os.path.dirname(SRC), "kara_q4.hip")).read()
    body = text[text.index("kara_status_t kara_q4_append("):text.index("kara_status_t kara_q4_read(")]
    launched = re.findall(r"hipLaunchKernelGGL\(\(?(q4_\w+_kernel)", body)
    # (few tokens: one launch for all of it)
    assert launched == ["q4_append_few_kernel", "q4_check_kernel", "q4_append_kernel", "q4_commit_kernel"]
    for name in ("q4_check_kernel", "q4_append_kernel"):
        params = re.search(name + r"\(\s*(Geom[^)]*)\)", text).group(1)
        assert re.search(r"const int32_t\* __restrict__ seq_lens", params), name
