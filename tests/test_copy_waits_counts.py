"""Waits for tile copies of the kernels with a key/value cache, by a count that holds for any number: a wait that allows n operations leaves
the n newest under way, and all of them where there are fewer. Read from the assembly hipcc makes of the kernels here."""
import re

import pytest

from test_copy_waits import _events, _kernels


def _left(under_way, n):
    return under_way[max(0, len(under_way) - n):]


def _reads_behind_copies(events, tile):
    """Transpose reads that come while a copy of V may be under way: tiles of `tile` copies each, K, V, K, V, ..."""
    copies, under_way, bad = 0, [], 0
    for e in events:
        if e == "copy":
            under_way.append("V" if copies // tile % 2 else "K")
            copies += 1
        elif e == "other":
            under_way.append("other")
        elif e == "read":
            bad += "V" in under_way
        else:
            under_way = _left(under_way, e)
    return bad, copies


def _barriers(lines):
    """Barriers, and how many of them a copy to LDS may be under way at."""
    under_way, barriers, bad = [], 0, 0
    for line in lines:
        s = line.strip()
        if re.match(r"(buffer|global|scratch)_(load|store)", s):
            under_way.append(" lds" in s)
        elif s.startswith("s_waitcnt") and "vmcnt" in s:
            under_way = _left(under_way, int(re.search(r"vmcnt\((\d+)\)", s).group(1)))
        elif s.startswith("s_barrier"):
            barriers += 1
            bad += any(under_way)
    return barriers, bad


def test_a_wait_that_allows_more_than_there_are():
    assert _left(list("abcdef"), 8) == list("abcdef") and _left(list("abcdef"), 6) == list("abcdef")
    assert _left(list("abcdef"), 2) == list("ef") and _left(list("abcdef"), 0) == [] and _left([], 3) == []
    # K and V of two copies each, then a wait that leaves all of them, and a read of V
    assert _reads_behind_copies(["copy"] * 4 + [8, "read"], 2) == (1, 4)
    assert _reads_behind_copies(["copy"] * 4 + [4, "read", 2, "read", 1, "read", 0, "read"], 2) == (3, 4)
    assert _reads_behind_copies(["copy"] * 4 + ["copy"] * 2 + [2, "read"], 2) == (0, 6)
    copy = "buffer_load_dwordx4 v1, s[0:3], 0 offen lds"
    assert _barriers([copy] * 6 + ["s_waitcnt vmcnt(8)", "s_barrier"]) == (1, 1)
    assert _barriers([copy] * 6 + ["s_waitcnt vmcnt(0)", "s_barrier", copy, "s_waitcnt vmcnt(1)", "s_barrier"]) == (2, 1)


def test_reads_of_the_barrier_free_loop(tmp_path_factory):
    kernels = _kernels("attn_paged.hip", r"few_rows_bf16_kernelILi(\d+)ELi\d+E", tmp_path_factory)
    assert len(kernels) == 6
    for D, body in kernels:
        bad, copies = _reads_behind_copies(_events(body), int(D) // 16)
        assert bad == 0 and copies > 0 and copies % (2 * (int(D) // 16)) == 0


def test_barriers_of_the_kernel_that_shares_its_tiles(tmp_path_factory):
    kernels = _kernels("attn_prompt_bf16.hip", r"prompt_bf16_kernelILi(\d+)E", tmp_path_factory)
    assert len(kernels) == 4
    for _, body in kernels:
        barriers, bad = _barriers(body.splitlines())
        assert bad == 0 and barriers >= 6
