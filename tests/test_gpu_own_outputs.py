"""Outputs that the calls of the denoising steps take for themselves, where the call runs on a stream that is not the current one: the
memory is not what the current stream still reads, and what the current stream reads of an output is there until it has."""
import pytest
import torch

import paper_2509_24014_amd as sd

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _busy(x):
    """Some 20 ms of work on the current stream."""
    for _ in range(20):
        x = x @ x * 1e-3
    return x


@pytest.mark.parametrize("which", ["dense", "dense_select", "sparse", "select"])
def test_on_another_stream(which):
    g = torch.Generator().manual_seed(1)
    q, q2, k, v = (torch.randn(1, 4, 512, 128, generator=g).to(torch.bfloat16).to(DEV) for _ in range(4))
    index = sd.select_pattern(q, k, 64, 64, 0.3)
    blocks = (64, 64, 0.3)
    call = {"dense": lambda q, **kw: sd.attn_dense(q, k, v, **kw), "sparse": lambda q, **kw: sd.attn_sparse(q, k, v, index, **kw),
            "dense_select": lambda q, **kw: sd.attn_dense_select(q, k, v, *blocks, **kw)[0],
            "select": lambda q, **kw: sd.select_pattern(q, k, *blocks, **kw).col_idx}[which]
    want, want2 = call(q).clone(), call(q2).clone()
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    load = torch.randn(4096, 4096, device=DEV)
    kept, kept_out = torch.zeros_like(want), torch.zeros_like(want)
    for _ in range(3):
        x = torch.full_like(want, 3)
        torch.cuda.synchronize()
        _busy(load)
        kept.copy_(x)                      # queued behind the load
        at = x.data_ptr()
        del x                              # the next block of this size that the current stream asks for
        out = call(q, stream=s)
        assert out.data_ptr() != at
        here.wait_stream(s)
        _busy(load)
        kept_out.copy_(out)
        del out
        again = call(q2, stream=s)         # written on s while `here` has yet to read the first
        torch.cuda.synchronize()
        assert (kept == 3).all() and torch.equal(kept_out, want) and torch.equal(again, want2)
        kept.zero_(), kept_out.zero_()
        del again
