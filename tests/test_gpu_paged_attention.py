"""The paged cache: append, attention of the newest tokens, the check of a page table, and all of them together as a program that
generates uses them. Attention against the formula in 64 bits, append exactly."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import attend64, check, make_cache, offsets, packed_reference, paged_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _paged(lens, new, Hq, Hkv, D, dtype, page, mask_block, seed=0, heads_first=False, extra=0, fill=math.nan):
    print(f"paged {new} of {lens}, heads {Hq}/{Hkv} of {D}, {dtype}, pages of {page}, blocks of {mask_block}", flush=True)
    kp, vp, table, seq_lens, rows = make_cache(lens, Hkv, D, dtype, page, seed, heads_first, fill=fill)
    g = torch.Generator().manual_seed(seed + 1)
    T = sum(new)
    q = torch.randn(T + extra, Hq, D, generator=g).to(dtype)
    out = torch.full((T + extra, Hq, D), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((Hq, T + extra), 7.0, device=DEV)
    cache = sd.PagedCache(kp, vp, table, seq_lens)
    cu = None if new == [1] * len(lens) and not extra else offsets(new, DEV)
    assert sd.attn_paged(q.to(DEV), cache, cu, mask_block=mask_block, out=out, lse_out=lse) is out
    torch.cuda.synchronize()
    assert (out[T:] == 7.0).all() and (lse[:, T:] == 7.0).all()
    check(out[:T], lse[:, :T], paged_reference(q, rows, new, mask_block), dtype, f"{lens} {new}")


LENGTHS = [[1], [15, 16, 17], [31, 33, 64], [0, 5, 0], [127, 128, 129], [255, 1, 257], [1000, 3], [40] * 9]
SETTINGS = [(BF, 128, 4, 2, 16), (BF, 64, 3, 3, 32), (F32, 128, 2, 1, 16), (F32, 64, 4, 4, 64), (BF, 128, 28, 4, 64), (BF, 64, 40, 2, 128),
            (F32, 128, 20, 1, 256), (BF, 128, 2, 2, 256)]


@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", SETTINGS)
def test_one_token(lens, dtype, D, Hq, Hkv, page):
    _paged(lens, [1] * len(lens), Hq, Hkv, D, dtype, page, 1, heads_first=page == 64)


# several new tokens: causal, a block in both directions, blocks that begin inside the new tokens, more new tokens than tokens
@pytest.mark.parametrize("lens,new", [([300, 40, 8], [5, 32, 8]), ([64, 100], [0, 33]), ([20, 500], [30, 1]), ([700], [130]), ([129, 0, 65], [65, 2, 65])], ids=str)
@pytest.mark.parametrize("mask_block", [1, 32, 7, 1 << 30])
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [(BF, 128, 4, 2, 16), (BF, 64, 3, 3, 32), (F32, 128, 2, 2, 32), (F32, 64, 6, 2, 16), (BF, 128, 14, 2, 128)])
def test_several_tokens(lens, new, mask_block, dtype, D, Hq, Hkv, page):
    _paged(lens, new, Hq, Hkv, D, dtype, page, mask_block, seed=3, heads_first=D == 64, extra=2)


@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf, 3e38], ids=str)
@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [(BF, 128, 4, 2, 16), (BF, 64, 2, 2, 64), (F32, 128, 2, 2, 16), (F32, 64, 2, 1, 32)])
def test_what_lies_behind_a_length_does_not_matter(fill, dtype, D, Hq, Hkv, page):
    _paged([1, 45, 100, 333], [1, 1, 1, 1], Hq, Hkv, D, dtype, page, 1, seed=4, fill=fill)
    _paged([33, 45, 100, 333], [9, 2, 30, 1], Hq, Hkv, D, dtype, page, 1, seed=5, fill=fill)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan], ids=str)
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_hidden_new_tokens_do_not_matter(dtype, D, bad):
    """Values of the later new tokens are not numbers or infinite: the earlier ones do not see them."""
    n, new = 150, 12
    kp, vp, table, seq_lens, rows = make_cache([n], 2, D, dtype, 16, 6)
    last = n - 5
    page = int(table[0, last // 16])
    vp[page, last % 16] = bad
    kp[page, last % 16] = bad
    q = torch.randn(new, 2, D, generator=torch.Generator().manual_seed(1)).to(dtype)
    lse = torch.empty(2, new, device=DEV)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets([new], DEV), lse_out=lse)
    want = attend64(q, *rows[0], 1)
    check(out[:7], lse[:, :7], tuple(w[:, :7] if i == 1 else w[:7] for i, w in enumerate(want)), dtype, str(bad))
    assert not torch.isfinite(out[7:]).any()


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,heads_first", [(BF, 128, 28, 4, 64, True), (BF, 64, 8, 8, 16, False), (F32, 128, 8, 2, 32, False)])
def test_long_and_short_sequences_of_a_batch(dtype, D, Hq, Hkv, page, heads_first):
    """The axis is split where it is long: parts of one sequence are joined, others are whole."""
    _paged([9000, 1, 130, 0, 4100, 2047], [1, 1, 1, 1, 1, 1], Hq, Hkv, D, dtype, page, 1, seed=7, heads_first=heads_first)
    _paged([5000, 40, 3], [17, 1, 3], Hq, Hkv, D, dtype, page, 4, seed=8, heads_first=heads_first)


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_that_climb_or_fall(dtype, D, sign):
    n = 2000
    kp, vp, table, seq_lens, rows = make_cache([n], 1, D, dtype, 16, 9)
    rows[0][0][:, :, 0] = (sign * torch.arange(n).float() * (0.0625 * D ** 0.5))[:, None].to(dtype)
    for t in range(n // 16):
        kp[int(table[0, t])] = rows[0][0][16 * t:16 * t + 16].to(DEV)
    q = torch.randn(1, 3, D, generator=torch.Generator().manual_seed(2)).to(dtype)
    q[:, :, 0] = 8.0
    lse = torch.empty(3, 1, device=DEV)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), lse_out=lse)
    check(out, lse, attend64(q, *rows[0], 1), dtype)


def test_many_sequences():
    """More sequences than a wave has lanes, some of them empty."""
    g = torch.Generator().manual_seed(3)
    lens = torch.randint(0, 90, (300,), generator=g).tolist()
    _paged(lens, [1] * 300, 4, 2, 64, BF, 16, 1, seed=10)
    new = [min(n, 3) if i % 3 else 0 for i, n in enumerate(lens)]
    _paged(lens, new, 2, 1, 64, F32, 32, 1, seed=11, extra=1)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page", [(BF, 128, 2, 1, 64), (F32, 64, 4, 4, 32), (BF, 64, 40, 2, 16)])
def test_many_sequences_of_which_some_are_split(dtype, D, Hq, Hkv, page):
    """Parts are counted over all sequences, 64 at a time."""
    lens = [5 + 7 * (i % 30) for i in range(150)]
    lens[3], lens[63], lens[64], lens[130], lens[149] = 3000, 1100, 2049, 900, 1500
    _paged(lens, [1] * 150, Hq, Hkv, D, dtype, page, 1, seed=20)
    new = [(3 if i in (3, 64, 149) else i % 2) for i in range(150)]
    _paged(lens, new, Hq, Hkv, D, dtype, page, 1, seed=21, extra=2)


def test_cache_of_more_than_32_bits():
    """Pages whose byte offsets, and whose element offsets, do not fit 32 bits."""
    H, D, page, n_pages = 16, 128, 64, 40000                                     # 10 GB each
    kp = torch.empty(n_pages, page, H, D, dtype=BF, device=DEV)
    vp = torch.empty(n_pages, page, H, D, dtype=BF, device=DEV)
    n = 130
    g = torch.Generator().manual_seed(12)
    k, v = torch.randn(n, H, D, generator=g).to(BF), torch.randn(n, H, D, generator=g).to(BF)
    q = torch.randn(1, H, D, generator=g).to(BF)
    table = torch.tensor([[n_pages - 1, n_pages // 2 + 7, 33000]], dtype=torch.int32, device=DEV)
    cache = sd.PagedCache(kp, vp, table, torch.tensor([n], dtype=torch.int32, device=DEV))
    sd.cache_append(cache, k.to(DEV), v.to(DEV), offsets([n], DEV))
    assert torch.equal(kp[n_pages - 1].cpu(), k[:64]) and torch.equal(vp[33000, :2].cpu(), v[128:])
    check(sd.attn_paged(q.to(DEV), cache), None, attend64(q, k, v, 1), BF)


# ------------------------------------------------------------------------------------------------ append


@pytest.mark.parametrize("dtype,D,H,page,heads_first", [(BF, 128, 4, 16, False), (BF, 64, 3, 32, True), (F32, 128, 2, 64, False), (F32, 64, 1, 256, True)])
@pytest.mark.parametrize("lens,new", [([1], [1]), ([20, 5, 100], [1, 1, 1]), ([70, 0, 33, 300], [70, 0, 1, 150]), ([10, 40], [30, 40])], ids=str)
def test_append(lens, new, dtype, D, H, page, heads_first):
    kp, vp, table, seq_lens, _ = make_cache(lens, H, D, dtype, page, 13, heads_first, fill=4.0)
    g = torch.Generator().manual_seed(14)
    T = sum(new)
    wide = torch.randn(T + 2, 2 * H + 1, D, generator=g).to(dtype)               # slices of one projection
    wide[0, 0, :3] = torch.tensor([math.nan, math.inf, -0.0]).to(dtype)
    dev = wide.to(DEV)
    want_k, want_v, at = kp.clone(), vp.clone(), 0
    for s, (m, n) in enumerate(zip(lens, new)):
        for i in range(n):
            pos = m - n + i
            if pos >= 0:
                want_k[int(table[s, pos // page]), pos % page] = dev[at + i, :H]
                want_v[int(table[s, pos // page]), pos % page] = dev[at + i, H:2 * H]
        at += n
    cache = sd.PagedCache(kp, vp, table, seq_lens)
    one_each = new == [1] * len(new)
    rows = T if one_each else T + 2                                              # two rows behind the last sequence
    k, v = dev[:rows, :H], dev[:rows, H:2 * H]
    assert sd.cache_append(cache, k, v, None if one_each else offsets(new, DEV)) is cache
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == BF else torch.int32
    assert torch.equal(kp.view(bits), want_k.view(bits)) and torch.equal(vp.view(bits), want_v.view(bits))


@pytest.mark.parametrize("tokens", [16383, 16384, 16500])
def test_append_past_the_caches(tokens):
    """64 MB of keys and values and more, the tokens of two sequences; attention then finds them."""
    H, D, page = 8, 128, 64
    n = [tokens - 5000, 5000]
    pages = [-(-x // page) for x in n]
    g = torch.Generator(device=DEV).manual_seed(23)
    k, v = (torch.randn(tokens, H, D, generator=g, device=DEV).to(BF) for _ in range(2))
    kp, vp = (torch.full((sum(pages), page, H, D), 3.0, dtype=BF, device=DEV) for _ in range(2))
    table = torch.zeros(2, max(pages), dtype=torch.int32, device=DEV)
    table[0, :pages[0]] = torch.arange(pages[0], device=DEV).flip(0)
    table[1, :pages[1]] = pages[0] + torch.arange(pages[1], device=DEV)
    lens = torch.tensor(n, dtype=torch.int32, device=DEV)
    cache = sd.cache_append(sd.PagedCache(kp, vp, table, lens), k, v, offsets(n, DEV))
    at = 0
    for s in range(2):
        for new, got in ((k, kp), (v, vp)):
            rows = got[table[s, :pages[s]].long()].flatten(0, 1)
            assert torch.equal(rows[:n[s]], new[at:at + n[s]]) and (rows[n[s]:] == 3.0).all()
        at += n[s]
    q = k[[n[0] - 1, tokens - 1]].contiguous()
    out = sd.attn_paged(q, cache)
    for s, rows in enumerate((slice(0, n[0]), slice(n[0], tokens))):
        check(out[s:s + 1], None, attend64(q[s:s + 1], k[rows], v[rows], 1), BF, f"sequence {s}")


def test_rows_outside_the_offsets_are_not_appended():
    kp, vp, table, seq_lens, _ = make_cache([50, 40], 2, 64, F32, 16, 17, fill=0.0)
    before = kp.clone()
    x = torch.ones(9, 2, 64, device=DEV)
    sd.cache_append(sd.PagedCache(kp, vp, table, seq_lens), x, x, offsets([4, 0, 2], DEV)[1:].contiguous())   # rows 4 and 5 of 9
    before[int(table[1, 2]), 6:8] = 1
    assert torch.equal(kp, before)


def test_page_numbers_out_of_range():
    """A wrong page is never written; the check finds it; the sequences beside it are as ever."""
    lens = [50, 40, 30]
    kp, vp, table, seq_lens, rows = make_cache(lens, 2, 64, BF, 16, 15, fill=0.0)
    cache = sd.PagedCache(kp, vp, table, seq_lens)
    sd.cache_validate(cache)                                                     # what lies behind a length is not looked at
    right = int(table[1, 1])
    for wrong in (-1, kp.shape[0], 2 ** 31 - 1, -2 ** 31):
        table[1, 1] = wrong
        with pytest.raises(sd.SparsedError) as e:
            sd.cache_validate(cache)
        assert e.value.status == 8
        before = kp.clone()
        x = torch.ones(20, 2, 64, dtype=BF, device=DEV)
        sd.cache_append(cache, x, x, offsets([0, 20, 0], DEV))                   # positions 20 .. 39 of sequence 1: page 1 and a half
        assert (kp[int(table[1, 2]), :8] == 1).all()
        kp.copy_(before)
        vp[int(table[1, 2]), :8] = rows[1][1][32:40].to(DEV)
        q = torch.randn(3, 2, 64, generator=torch.Generator().manual_seed(1)).to(BF)
        out = sd.attn_paged(q.to(DEV), cache)
        for s in (0, 2):
            check(out[s:s + 1], None, attend64(q[s:s + 1], *rows[s], 1), BF)
    table[1, 1] = right
    sd.cache_validate(cache)
    for wrong in (-1, 16 * table.shape[1] + 1):
        seq_lens[2] = wrong
        with pytest.raises(sd.SparsedError):
            sd.cache_validate(cache)
        sd.attn_paged(q.to(DEV), cache)                                          # cut to what the table can name
        torch.cuda.synchronize()


# ------------------------------------------------------------------------------------------------ together


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,block", [(BF, 128, 4, 2, 16, 1), (F32, 64, 2, 2, 32, 1), (BF, 64, 6, 2, 64, 32), (F32, 128, 4, 1, 16, 8)])
def test_prompts_then_blocks_of_new_tokens(dtype, D, Hq, Hkv, page, block):
    """A batch of prompts, then steps of `block` new tokens: what every step gives is what attention of the whole sequence
    gives at those rows."""
    g = torch.Generator().manual_seed(16)
    prompts, steps = [3 * block + 2, 70, 1], 4
    # sequences end on block edges after the first step, as a program that generates blocks keeps them
    first = [(-n) % block or block for n in prompts]
    total = [n + f + (steps - 1) * block for n, f in zip(prompts, first)]
    q, k, v = ([torch.randn(n, h, D, generator=g).to(dtype) for n in total] for h in (Hq, Hkv, Hkv))
    want = [attend64(a, b, c, block) for a, b, c in zip(q, k, v)]
    counts = [-(-n // page) for n in total]
    shape = (sum(counts) + 1, page, Hkv, D)
    kp, vp = (torch.full(shape, math.nan, dtype=dtype, device=DEV) for _ in range(2))
    table = torch.zeros(3, max(counts), dtype=torch.int32)
    pages = torch.randperm(shape[0], generator=g).tolist()
    for s, n in enumerate(counts):
        for t in range(n):
            table[s, t] = pages.pop()
    lens = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    cache = sd.PagedCache(kp, vp, table.to(DEV), lens)
    cat = lambda xs, at, n: torch.cat([x[a:a + c] for x, a, c in zip(xs, at, n)]).to(DEV)
    at, n = [0, 0, 0], prompts
    cu = offsets(n, DEV)
    kn, vn = cat(k, at, n), cat(v, at, n)
    out = sd.attn_prompt(cat(q, at, n), kn, vn, cu, mask_block=block)
    check(out, None, packed_reference(torch.cat([x[:c] for x, c in zip(q, n)]), torch.cat([x[:c] for x, c in zip(k, n)]),
                                      torch.cat([x[:c] for x, c in zip(v, n)]), n, n, block), dtype, "prompts")
    sd.cache_append(cache, kn, vn, cu)
    at = list(n)
    for step in range(steps):
        n = first if step == 0 else [block] * 3
        lens += torch.tensor(n, dtype=torch.int32, device=DEV)
        cu = None if n == [1, 1, 1] else offsets(n, DEV)
        sd.cache_append(cache, cat(k, at, n), cat(v, at, n), cu)
        lse = torch.empty(Hq, sum(n), device=DEV)
        out = sd.attn_paged(cat(q, at, n), cache, cu, mask_block=block, lse_out=lse)
        rows = tuple(torch.cat([(w[i][:, a:a + c] if i == 1 else w[i][a:a + c]) for w, a, c in zip(want, at, n)], 1 if i == 1 else 0) for i in range(4))
        check(out, lse, rows, dtype, f"step {step}")
        at = [a + c for a, c in zip(at, n)]
    sd.cache_validate(cache)


def test_steps_replayed_from_a_graph():
    """Append and attention of one token each, captured once: lengths and new rows change in place between replays; every replay
    gives what the eager calls give. Two graphs have a workspace each."""
    D, Hq, Hkv, page, B = 128, 8, 2, 16, 3
    lens0 = [40, 1500, 7]
    table = torch.randperm(400, generator=torch.Generator().manual_seed(4))[:300].view(3, 100).to(torch.int32).to(DEV)
    lens = torch.tensor(lens0, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(5)
    kp, vp = (torch.randn(400, page, Hkv, D, device=DEV, generator=g).to(BF) for _ in range(2))
    cache = sd.PagedCache(kp, vp, table, lens)
    q, k, v = (torch.randn(B, h, D, device=DEV, generator=g).to(BF) for h in (Hq, Hkv, Hkv))
    need = sd.paged_workspace_bytes(q, cache)
    out = [torch.empty_like(q) for _ in range(2)]
    graphs, spaces = [], [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o, ws in zip(out, spaces):
        with torch.cuda.stream(side):
            sd.attn_paged(q, cache, out=o, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            sd.cache_append(cache, k, v)
            sd.attn_paged(q, cache, out=o, workspace=ws)
        graphs.append(graph)
    for step in range(6):
        lens += 1 if step % 2 else 33
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device=DEV, generator=g).to(BF))
        graphs[step % 2].replay()
        torch.cuda.synchronize()
        got = out[step % 2].clone()
        sd.cache_append(cache, k, v)
        want = sd.attn_paged(q, cache)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_two_calls_at_once():
    """Two streams, a workspace each (one the call's own): each gives what it gives alone."""
    lens = [3000, 100]
    kp, vp, table, seq_lens, _ = make_cache(lens, 4, 128, BF, 32, 17)
    cache = sd.PagedCache(kp, vp, table, seq_lens)
    g = torch.Generator().manual_seed(6)
    qs = [torch.randn(2, 8, 128, generator=g).to(BF).to(DEV) for _ in range(2)]
    alone = [sd.attn_paged(q, cache) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [sd.attn_paged(q, cache, stream=s) for q, s in zip(qs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(alone, got))


@pytest.mark.parametrize("new,mask_block", [(1, 1), (9, 1), (9, 32), (9, 100), (40, 32)])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_last_value_is_infinite(dtype, D, new, mask_block):
    """The rows that see the last token show an infinity; what lies behind it in its page takes no part, nor does it in other rows."""
    n = 141
    kp, vp, table, seq_lens, rows = make_cache([n], 2, D, dtype, 16, 18)
    vp[int(table[0, 140 // 16]), 140 % 16] = math.inf
    q = torch.randn(new, 2, D, generator=torch.Generator().manual_seed(3)).to(dtype)
    out = sd.attn_paged(q.to(DEV), sd.PagedCache(kp, vp, table, seq_lens), offsets([new], DEV), mask_block=mask_block)
    want = attend64(q, *rows[0], mask_block)
    hidden = max(0, 140 // mask_block * mask_block - (n - new))
    if hidden:
        check(out[:hidden], None, tuple(w[:, :hidden] if i == 1 else w[:hidden] for i, w in enumerate(want)), dtype)
    assert (out[hidden:] == math.inf).all()
