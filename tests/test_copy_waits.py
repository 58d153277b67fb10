"""Waits for tile copies (global -> LDS) of the kernels with a key/value cache, read from the assembly hipcc makes of them here. The
compiler does not see that a transpose read needs a copy, so each wait is written out, or is that of a barrier."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_24014_amd import build as lib_build

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def _kernels(source, pattern, tmp_path_factory):
    if not (os.path.exists(HIPCC) or shutil.which(HIPCC)):
        pytest.skip("no hipcc here")
    out = str(tmp_path_factory.mktemp("asm") / "kernels.s")
    subprocess.run([HIPCC, *lib_build.FLAGS, "-S", "--cuda-device-only", os.path.join(lib_build.CSRC, source), "-o", out],
                   check=True, capture_output=True, timeout=300)
    with open(out) as f:
        return re.findall(r"^_ZN7sparsed\d+" + pattern + r"\w*:(.*?)^\.Lfunc_end", f.read(), re.M | re.S)


@pytest.fixture(scope="module")
def few_rows(tmp_path_factory):
    return _kernels("attn_paged.hip", r"few_rows_bf16_kernelILi(\d+)ELi\d+E", tmp_path_factory)


def _events(body):
    """Copies ("copy"), transpose reads ("read") and waits (how many loads they leave) in the order of the text, from loop heads on."""
    for line in body.splitlines():
        s = line.strip()
        if re.match(r"buffer_load_dwordx4 .* lds", s):
            yield "copy"
        elif s.startswith(("global_load", "buffer_load", "scratch_load", "global_store", "buffer_store", "scratch_store")):
            yield "other"
        elif s.startswith("ds_read_b64_tr"):
            yield "read"
        elif s.startswith("s_waitcnt") and "vmcnt" in s:
            yield int(re.search(r"vmcnt\((\d+)\)", s).group(1))


def test_counted_waits_of_the_barrier_free_loop(few_rows):
    """A step leaves the copy of one tile (D / 16 loads of a wave) under way at each of its waits. Tiles are copied K, V, K, V, ...; no
    transpose read, which is one of V, comes while a copy of V may be under way."""
    assert len(few_rows) == 6
    for D, body in few_rows:
        tile = int(D) // 16
        written = [int(n) for n in re.findall(r"#ASMSTART\s+s_waitcnt vmcnt\((\d+)\)", body)]
        assert set(written) <= {0, tile} and written.count(tile) >= 3, written
        copies, under_way = 0, []
        for e in _events(body):
            if e == "copy":
                under_way.append("V" if copies // tile % 2 else "K")
                copies += 1
            elif e == "other":
                under_way.append("other")
            elif e == "read":
                assert "V" not in under_way
            else:
                under_way = under_way[len(under_way) - e:] if e else []
        assert copies % (2 * tile) == 0


def test_barriers_wait_for_every_copy(tmp_path_factory):
    """In the kernel whose waves share their tiles a copy is waited for at the barrier behind it."""
    kernels = _kernels("attn_prompt_bf16.hip", r"prompt_bf16_kernelILi(\d+)E", tmp_path_factory)
    assert len(kernels) == 4
    for body in kernels:
        under_way, barriers = [], 0   # vector memory operations in the order of the text, which is that of execution between barriers
        for line in body[1].splitlines():
            s = line.strip()
            if re.match(r"(buffer|global|scratch)_(load|store)", s):
                under_way.append(" lds" in s)
            elif s.startswith("s_waitcnt") and "vmcnt" in s:
                n = int(re.search(r"vmcnt\((\d+)\)", s).group(1))
                under_way = under_way[len(under_way) - n:] if n else []
            elif s.startswith("s_barrier"):
                assert not any(under_way)
                barriers += 1
        assert barriers >= 6
