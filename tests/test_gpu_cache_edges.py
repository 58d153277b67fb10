"""Edges of the paged cache's calls: lengths beyond the page table, tables and streams that are not the plain ones."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import attend64, check, make_cache, offsets, paged_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


# ------------------------------------------------------------------------------------------------ lengths beyond the table


@pytest.mark.parametrize("dtype,D,page", [(BF, 128, 16), (F32, 64, 32)])
@pytest.mark.parametrize("beyond,new", [(1, 1), (1, 5), (7, 5), (5, 5), (40, 64), (2 ** 31 - 65, 3), (-66, 2), (-2 ** 31 - 64, 2)])
def test_append_behind_the_last_page(dtype, D, page, beyond, new):
    """The table of a sequence names 64 tokens and its length is 64 + beyond: tokens with a place go there, the others nowhere; the pages
    of the sequence, and those of the one beside it, keep the rest bit for bit."""
    print(f"append {new} tokens up to {64 + beyond} of 64, {dtype}", flush=True)
    kp, vp, table, lens, _ = make_cache([64, 20], 2, D, dtype, page, 30, fill=4.0, room=0)
    lens[0] = 64 + beyond
    g = torch.Generator().manual_seed(31)
    k, v = (torch.randn(new + 1, 2, D, generator=g).to(dtype).to(DEV) for _ in range(2))
    want_k, want_v = kp.clone(), vp.clone()
    places = [(0, 64 + beyond - new + i, i) for i in range(new)] + [(1, 19, new)]
    for s, pos, i in places:
        if 0 <= pos < 64:
            want_k[int(table[s, pos // page]), pos % page], want_v[int(table[s, pos // page]), pos % page] = k[i], v[i]
    cache = sd.PagedCache(kp, vp, table, lens)
    sd.cache_append(cache, k, v, None if new == 1 else offsets([new, 1], DEV))
    torch.cuda.synchronize()
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)
    with pytest.raises(sd.SparsedError):
        sd.cache_validate(cache)
