"""Edges of the calls with a key/value cache: lengths beyond the page table, streams, offsets outside the array, weights in two parts, sequences
continued by many tokens or few, tables that are not the plain ones."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import U32, UBF, attend64, check, make_cache, offsets, paged_reference

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


# ------------------------------------------------------------------------------------------------ streams


def _calls(H=8, D=128):
    """Both attention calls at one size: the call, its q, and what it gives."""
    g = torch.Generator().manual_seed(32)
    n = [300, 212]
    kp, vp, table, lens, _ = make_cache(n, 2, D, BF, 64, 33, fill=0.0)
    k, v = (torch.randn(sum(n), 2, D, generator=g).to(BF).to(DEV) for _ in range(2))
    cu, cache = offsets(n, DEV), sd.PagedCache(kp, vp, table, lens)
    qs = [torch.randn(sum(n), H, D, generator=g).to(BF).to(DEV) for _ in range(2)]
    return [(lambda q, **kw: sd.attn_prompt(q, k, v, cu, **kw), qs), (lambda q, **kw: sd.attn_paged(q, cache, cu, **kw), qs)]


def _busy(x):
    """Some 20 ms of work on the current stream."""
    for _ in range(20):
        x = x @ x * 1e-3
    return x


@pytest.mark.parametrize("which", [0, 1], ids=["prompt", "paged"])
def test_own_output_on_another_stream(which):
    """The output that a call takes for itself on stream s is not memory that the current stream still reads, and what the current
    stream reads of it is there until it has."""
    call, (q, q2) = _calls()[which]
    want, want2 = call(q), call(q2)
    s, here = torch.cuda.Stream(), torch.cuda.current_stream()
    load = torch.randn(4096, 4096, device=DEV)
    kept, kept_out = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    for _ in range(3):
        x = torch.full_like(q, 3.0)
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
        assert (kept == 3.0).all() and torch.equal(kept_out, want) and torch.equal(again, want2)
        kept.zero_(), kept_out.zero_()
        del again


# ------------------------------------------------------------------------------------------------ offsets


# forms of a prompt call: 32 rows a work-group, 128, 256; fp32 16 and 32
@pytest.mark.parametrize("dtype,Hq,Hkv,T", [(BF, 4, 2, 400), (BF, 48, 8, 400), (BF, 176, 22, 800), (F32, 4, 2, 400), (F32, 48, 8, 400)])
def test_offsets_outside_the_array_count_as_its_ends(dtype, Hq, Hkv, T):
    """Below 0 and beyond L, ascending: the same bits as with 0 and L."""
    g = torch.Generator(device=DEV).manual_seed(34)
    q, k, v = (torch.randn(T, h, 128, generator=g, device=DEV).to(dtype) for h in (Hq, Hkv, Hkv))
    for wild, cut in (([-2 ** 31, -5, 150, 2 ** 31 - 1], [0, 0, 150, T]), ([-1, T + 1, T + 2, 2 ** 30], [0, T, T, T]), ([-9, 130, T, T + 7], [0, 130, T, T])):
        got = []
        for cu in (wild, cut):
            out, lse = torch.full_like(q, 9.0), torch.full((Hq, T), 9.0, device=DEV)
            sd.attn_prompt(q, k, v, torch.tensor(cu, dtype=torch.int32, device=DEV), out=out, lse_out=lse)
            got.append((out, lse))
        torch.cuda.synchronize()
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
        assert torch.isfinite(got[0][0]).all() and (got[0][0] != 9.0).any(2).all()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_offsets_outside_the_array_in_a_cache(dtype, D):
    lens = [900, 30, 70]
    for wild, cut in (([-3, 5, 20, 2 ** 31 - 1], [0, 5, 20, 41]), ([-2 ** 31, -1, 41, 60], [0, 0, 41, 41])):
        got = []
        for cu in (wild, cut):
            kp, vp, table, seq_lens, _ = make_cache(lens, 2, D, dtype, 32, 35, fill=0.0)
            g = torch.Generator(device=DEV).manual_seed(36)
            q, k, v = (torch.randn(41, h, D, generator=g, device=DEV).to(dtype) for h in (4, 2, 2))
            cu, cache, out = torch.tensor(cu, dtype=torch.int32, device=DEV), sd.PagedCache(kp, vp, table, seq_lens), torch.full_like(q, 9.0)
            sd.cache_append(cache, k, v, cu)
            sd.attn_paged(q, cache, cu, out=out)
            got.append((kp, vp, out))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(*got))
        assert torch.isfinite(got[0][2]).all() and (got[0][2] != 9.0).any(2).all()


def test_validation_of_more_sequences_than_a_launch_has_work_groups():
    n = (1 << 24) + 5
    pages = torch.zeros(3, 16, 1, 64, dtype=BF, device=DEV)
    table, lens = torch.zeros(n, 1, dtype=torch.int32, device=DEV), torch.full((n,), 16, dtype=torch.int32, device=DEV)
    cache = sd.PagedCache(pages, pages, table, lens)
    sd.cache_validate(cache)
    for s in (0, 65536, n - 1):
        for t, bad in ((table[:, 0], 3), (lens, 17)):
            was = int(t[s])
            t[s] = bad
            with pytest.raises(sd.SparsedError) as e:
                sd.cache_validate(cache)
            assert e.value.status == 8
            t[s] = was
    sd.cache_validate(cache)


# ------------------------------------------------------------------------------------------------ probabilities in two parts


@pytest.mark.parametrize("lens,new,Hq,Hkv,D", [([5, 33, 700], [1, 1, 1], 8, 2, 128), ([3000], [1], 28, 4, 128), ([257, 64], [4, 4], 8, 2, 64), ([1500, 9, 40], [2, 1, 2], 3, 3, 64)], ids=str)
def test_weights_are_not_rounded_to_one_part(lens, new, Hq, Hkv, D):
    """Up to 16 rows a sequence and key/value head. A weight is off by half a step of half a step, 2^-16 of itself, in the product with V; what else there
    is, is fp32 (cache_utils) and the rounding of the result, 2^-8 of itself."""
    kp, vp, table, seq_lens, rows = make_cache(lens, Hkv, D, BF, 32, 37)
    q = torch.randn(sum(new), Hq, D, generator=torch.Generator().manual_seed(38)).to(BF)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets(new, DEV))
    want, _, A, rel = paged_reference(q, rows, new, 1)
    bound = A * (2.0 * rel[..., None] + 8 * U32 + UBF * UBF) + UBF * want.abs() + 2.0 ** -126
    assert ((out.double().cpu() - want).abs() <= bound).all(), ((out.double().cpu() - want).abs() - bound).max()


@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan], ids=str)
@pytest.mark.parametrize("D,where", [(128, 3), (64, 3), (128, 70), (64, 950)])
def test_an_infinite_value_that_every_row_sees(D, where, bad, new):
    """It is that of the result, whatever the parts of its weight are, and only in its column and head."""
    n = 1000
    kp, vp, table, seq_lens, rows = make_cache([n], 2, D, BF, 16, 39)
    vp[int(table[0, where // 16]), where % 16, 1, 5] = bad
    q = torch.randn(new, 4, D, generator=torch.Generator().manual_seed(41)).to(BF)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets([new], DEV))
    got = out[:, 2:, 5].float()
    assert (torch.isnan(got).all() if math.isnan(bad) else (got == bad).all())
    clean = out.clone()
    clean[:, 2:, 5] = 0
    want, lse, A, rel = attend64(q, *rows[0], 1)
    want[:, 2:, 5], A[:, 2:, 5] = 0, 0
    check(clean, None, (want, lse, A, rel), BF)


# ------------------------------------------------------------------------------------------------ continued sequences, other tables


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [(BF, 128, 4, 2, 64), (BF, 64, 8, 2, 16), (F32, 128, 2, 1, 32)])
@pytest.mark.parametrize("lens,new,mask_block", [([2100, 300], [300, 300], 1), ([1500, 40, 700], [257, 1, 130], 32)], ids=str)
def test_a_chunk_of_hundreds_of_tokens(lens, new, mask_block, dtype, D, Hq, Hkv, page):
    kp, vp, table, seq_lens, rows = make_cache(lens, Hkv, D, dtype, page, 42)
    q = torch.randn(sum(new), Hq, D, generator=torch.Generator().manual_seed(43)).to(dtype)
    lse = torch.empty(Hq, sum(new), device=DEV)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets(new, DEV), mask_block=mask_block, lse_out=lse)
    check(out, lse, paged_reference(q, rows, new, mask_block), dtype)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,lens", [(F32, 128, 8, 2, [20000, 3]), (F32, 64, 4, 4, [6000, 9001, 12])])
def test_long_fp32_caches(dtype, D, Hq, Hkv, lens):
    kp, vp, table, seq_lens, rows = make_cache(lens, Hkv, D, dtype, 64, 44)
    q = torch.randn(len(lens), Hq, D, generator=torch.Generator().manual_seed(45)).to(dtype)
    lse = torch.empty(Hq, len(lens), device=DEV)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), lse_out=lse)
    check(out, lse, paged_reference(q, rows, [1] * len(lens), 1), dtype)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,n_q", [(BF, 128, 28, 4, 1), (BF, 64, 8, 2, 9), (F32, 128, 4, 1, 5)])
def test_few_queries_over_long_packed_keys(dtype, D, Hq, Hkv, n_q):
    """As a prompt call, and as a paged call over the same memory seen as pages of 64 tokens."""
    g = torch.Generator().manual_seed(46)
    n_k = [64 * 150, 64 * 3]
    T = sum(n_k)
    k, v = (torch.randn(T, Hkv, D, generator=g).to(dtype) for _ in range(2))
    q = torch.randn(2 * n_q, Hq, D, generator=g).to(dtype)
    dev, cu_q = [x.to(DEV) for x in (q, k, v)], offsets([n_q, n_q], DEV)
    want = paged_reference(q, [(k[:n_k[0]], v[:n_k[0]]), (k[n_k[0]:], v[n_k[0]:])], [n_q, n_q], 1)
    lse = torch.empty(Hq, 2 * n_q, device=DEV)
    check(sd.attn_prompt(*dev, cu_q, offsets(n_k, DEV), lse_out=lse), lse, want, dtype, "prompt")
    table = torch.zeros(2, 150, dtype=torch.int32, device=DEV)
    table[0], table[1, :3] = torch.arange(150), torch.arange(150, 153)
    cache = sd.PagedCache(*(x.view(-1, 64, Hkv, D) for x in dev[1:]), table, torch.tensor(n_k, dtype=torch.int32, device=DEV))
    check(sd.attn_paged(dev[0], cache, cu_q, lse_out=lse), lse, want, dtype, "paged")


@pytest.mark.parametrize("dtype,D", [(BF, 128), (F32, 64)])
def test_page_table_cut_from_a_wider_one(dtype, D):
    """Rows further apart than they are long, the first entry not the first of its memory."""
    lens = [900, 30, 70]
    kp, vp, table, seq_lens, rows = make_cache(lens, 2, D, dtype, 32, 47)
    wide = torch.full((4, table.shape[1] + 9), -7, dtype=torch.int32, device=DEV)
    wide[1:, 5:5 + table.shape[1]] = table
    cut = wide[1:, 5:5 + table.shape[1]]
    assert not cut.is_contiguous()
    q, k, v = (torch.randn(3, h, D, generator=torch.Generator().manual_seed(48 + i)).to(dtype) for i, h in enumerate((4, 2, 2)))
    cache = sd.PagedCache(kp, vp, cut, seq_lens)
    sd.cache_validate(cache)
    sd.cache_append(cache, k.to(DEV), v.to(DEV))                                 # in place of every last token
    for s, n in enumerate(lens):
        rows[s][0][n - 1], rows[s][1][n - 1] = k[s], v[s]
    check(sd.attn_paged(q.to(DEV), cache), None, paged_reference(q, rows, [1, 1, 1], 1), dtype)


# ------------------------------------------------------------------------------------------------ the range of logits


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("dtype,D,Hq,Hkv", [(BF, 128, 8, 2), (BF, 64, 4, 4), (F32, 128, 2, 2), (F32, 64, 4, 2)])
@pytest.mark.parametrize("q0,k0", [((1 + 11 / 128) * 2.0 ** 60, -(1 + 23 / 128) * 2.0 ** 60), ((1 + 11 / 128) * 2.0 ** 60, (1 + 23 / 128) * 2.0 ** 60),
                                   ((1 + 11 / 128) * 2.0 ** 20, -(1 + 23 / 128) * 2.0 ** 18), ((1 + 11 / 128) * 2.0 ** 20, (1 + 23 / 128) * 2.0 ** 18)], ids=str)
def test_equal_logits_of_any_size(dtype, D, Hq, Hkv, q0, k0, new):
    """Keys are one column, all the same: a row is the mean of the values it sees, its log-sum-exp the logit and log n. Bounds as in the test
    of the same name for prompts."""
    n = 1200
    kp, vp, table, seq_lens, rows = make_cache([n], Hkv, D, dtype, 64, 50)
    kp.zero_()[..., 0] = k0
    q = torch.zeros(new, Hq, D, dtype=dtype)
    q[..., 0] = q0
    lse = torch.empty(Hq, new, device=DEV)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets([new], DEV), lse_out=lse).double().cpu()
    v = rows[0][1].double().repeat_interleave(Hq // Hkv, 1)
    logit = float(q[0, 0, 0]) * float(kp[0, 0, 0, 0]) / math.sqrt(D)
    for i in range(new):
        seen = n - new + i + 1
        A, want = v[:seen].abs().mean(0), v[:seen].mean(0)
        assert ((out[i] - want).abs() <= ((2 * UBF if dtype == BF else 2 * U32) + (seen + 8) * U32) * A).all()
        assert ((lse[:, i].double().cpu() - (logit + math.log(seen))).abs() <= 8 * U32 * abs(logit) + (seen + 8) * U32).all()
