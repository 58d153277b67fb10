"""Attention of packed prompts (attn_prompt) against the formula in 64 bits: lengths around every tile edge, both types, grouped
heads, masks in blocks, strided views, rows that see nothing, what lies behind the last sequence, values that a mask hides."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import check, offsets, packed_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


def _rows(T, H, D, dtype, g, scale=1.0):
    return (torch.randn(T, H, D, generator=g) * scale).to(dtype)


def _run(n_q, n_k, Hq, Hkv, D, dtype, mask_block, seed=0, scale=1.0, extra=0, edit=None):
    print(f"prompt {n_q} over {n_k if n_k else 'own keys'}, heads {Hq}/{Hkv} of {D}, {dtype}, blocks of {mask_block}", flush=True)
    g = torch.Generator().manual_seed(seed)
    T, Tk = sum(n_q), sum(n_k or n_q)
    q = _rows(T + extra, Hq, D, dtype, g, scale)
    k, v = _rows(Tk + extra, Hkv, D, dtype, g, scale), _rows(Tk + extra, Hkv, D, dtype, g)
    if edit is not None:
        edit(q, k, v)
    out = torch.full((T + extra, Hq, D), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((Hq, T + extra), 7.0, device=DEV)
    cu_q = offsets(n_q, DEV)
    cu_k = None if n_k is None else offsets(n_k, DEV)
    got = sd.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu_q, cu_k, mask_block=mask_block, out=out, lse_out=lse)
    torch.cuda.synchronize()
    assert got is out
    assert (out[T:] == 7.0).all() and (lse[:, T:] == 7.0).all()      # behind the last sequence
    return q, k, v, out[:T], lse[:, :T]


LENGTHS = [[1], [2, 1], [31, 32, 33], [63, 1, 65], [127, 0, 129], [64, 64], [0, 5, 0, 0, 300], [257, 40], [513], [100] * 5]


@pytest.mark.parametrize("n", LENGTHS, ids=str)
@pytest.mark.parametrize("dtype,D,Hq,Hkv,mask_block", [(BF, 128, 4, 2, 1), (BF, 64, 3, 3, 1), (F32, 128, 2, 1, 1), (F32, 64, 4, 2, 32),
                                                      (BF, 128, 2, 2, 32), (BF, 64, 7, 1, 5), (F32, 128, 3, 3, 100)])
def test_lengths_around_tile_edges(n, dtype, D, Hq, Hkv, mask_block):
    q, k, v, out, lse = _run(n, None, Hq, Hkv, D, dtype, mask_block, extra=3)
    check(out, lse, packed_reference(q, k, v, n, n, mask_block), dtype, str(n))


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_block_that_hides_nothing(dtype, D):
    n = [70, 200, 1]
    q, k, v, out, lse = _run(n, None, 2, 2, D, dtype, 2 ** 31 - 1)
    check(out, lse, packed_reference(q, k, v, n, n, 1 << 30), dtype)
    want = sd.attn_dense(q[None, 70:270].transpose(1, 2).to(DEV), k[None, 70:270].transpose(1, 2).to(DEV), v[None, 70:270].transpose(1, 2).to(DEV))
    d = (want[0].transpose(0, 1).double() - out[70:270].double()).abs().max().item()
    assert d <= (2.0 ** -5 if dtype == BF else 1e-5)       # the framework's own dense call


# queries that are the last tokens of longer key sequences, and of shorter ones: rows that see nothing
@pytest.mark.parametrize("n_q,n_k", [([5, 64, 1], [300, 64, 129]), ([40, 3], [10, 0]), ([130, 0, 65], [131, 50, 1]), ([1, 1, 1], [1, 1000, 64])], ids=str)
@pytest.mark.parametrize("dtype,D,mask_block", [(BF, 128, 1), (BF, 64, 16), (F32, 128, 1), (F32, 64, 32)])
def test_other_key_lengths(n_q, n_k, dtype, D, mask_block):
    q, k, v, out, lse = _run(n_q, n_k, 4, 2, D, dtype, mask_block, seed=4, extra=2)
    check(out, lse, packed_reference(q, k, v, n_q, n_k, mask_block), dtype)


def test_no_keys_at_all():
    for dtype in (BF, F32):
        q = torch.randn(6, 2, 64, device=DEV).to(dtype)
        k = torch.empty(0, 1, 64, dtype=dtype, device=DEV)
        lse = torch.zeros(2, 6, device=DEV)
        out = sd.attn_prompt(q, k, k, offsets([4, 2], DEV), offsets([0, 0], DEV), lse_out=lse)
        assert (out == 0).all() and (lse == -math.inf).all()
        assert sd.attn_prompt(q[:0], k, k, offsets([0], DEV)).shape == (0, 2, 64)
        kept = torch.full_like(q, 3.0)
        sd.attn_prompt(q, q[:, :1], q[:, :1], offsets([], DEV), out=kept)
        assert (kept == 3.0).all()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_strided_views(dtype, D):
    """q, k, v as slices of one projection, output heads first: nothing but the last dimension is contiguous."""
    g = torch.Generator().manual_seed(5)
    n, Hq, Hkv = [150, 33], 6, 2
    T = sum(n)
    qkv = torch.randn(T, Hq + 2 * Hkv + 1, D, generator=g).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:Hq + 2 * Hkv]
    dev = qkv.to(DEV)
    out = torch.full((Hq, T, D), 5.0, dtype=dtype, device=DEV)
    lse = torch.empty(Hq, T, device=DEV)
    sd.attn_prompt(dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:Hq + 2 * Hkv], offsets(n, DEV), out=out.transpose(0, 1), lse_out=lse)
    check(out.transpose(0, 1), lse, packed_reference(q, k, v, n, n, 1), dtype)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan], ids=str)
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_hidden_places_do_not_matter(dtype, D, bad):
    """Keys and values at and behind a token are not numbers or infinite: rows before it are as if they were not there."""
    n, cut = [90, 200, 40], 90 + 77

    def edit(q, k, v):
        k[cut], v[cut + 1] = bad, bad
        k[-3:], v[-3:] = bad, bad

    q, k, v, out, lse = _run(n, None, 2, 1, D, dtype, 1, seed=6, extra=3, edit=edit)
    clean = _run(n, None, 2, 1, D, dtype, 1, seed=6, extra=3)
    want = packed_reference(clean[0], clean[1], clean[2], n, n, 1)
    for rows in (slice(0, cut), slice(290, 330)):
        check(out[rows], lse[:, rows], tuple(w[:, rows] if i == 1 else w[rows] for i, w in enumerate(want)), dtype, f"{bad} rows {rows}")
    # a row that sees it shows it: the value cut + 1 is seen by row cut + 1 and those after it in the sequence
    assert not torch.isfinite(out[cut + 1:290]).any()


@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_that_climb_or_fall(dtype, D, sign):
    """Logits that leave the range of the first keys by hundreds of octaves along the sequence."""
    n = [400, 130]

    def edit(q, k, v):
        q[:, :, 0] = 8.0
        ramp = torch.arange(k.shape[0]).float() * (0.125 * D ** 0.5)
        k[:, :, 0] = (sign * ramp)[:, None].to(dtype)

    q, k, v, out, lse = _run(n, None, 2, 2, D, dtype, 1, seed=7, edit=edit)
    check(out, lse, packed_reference(q, k, v, n, n, 1), dtype)


def test_masked_logits_of_the_lowest_value():
    """-3.4e38 as a logit (a key far against the query) is a weight of zero, not a row without weight."""
    for dtype in (BF, F32):
        def edit(q, k, v):
            q[:, :, 0] = 2.0 ** 60
            k[:, :, 0] = 0.0
            k[3:, :, 0] = -2.0 ** 66

        q, k, v, out, lse = _run([80], None, 2, 2, 64, dtype, 1, seed=8, edit=edit)
        want = packed_reference(q, k, v, [80], [80], 1)
        # from row 3 on the first three keys have all of the weight
        d = (out.double().cpu() - want[0]).abs()
        assert torch.isfinite(out).all() and d.max() <= (2.0 ** -5 if dtype == BF else 1e-4)


def test_offsets_out_of_range_stay_inside():
    """Offsets that descend or leave the array are cut; rows that sound offsets name are as ever."""
    for dtype, D in ((BF, 128), (F32, 64)):
        g = torch.Generator().manual_seed(9)
        q, k, v = (torch.randn(100, 2, D, generator=g).to(dtype) for _ in range(3))
        cu = torch.tensor([0, 60, 1000, -7], dtype=torch.int32, device=DEV)       # 0-60, 60-100, nothing
        out = torch.full((100, 2, D), 9.0, dtype=dtype, device=DEV)
        sd.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), cu, out=out)
        torch.cuda.synchronize()
        want = packed_reference(q, k, v, [60], [60], 1)
        check(out[:60], None, want, dtype)


def test_rows_beyond_32_bit_offsets():
    """A packed array of more than 2^32 bytes: the rows at its end."""
    T, H, D = 70000, 256, 128                                                    # 4.6 GB
    k = torch.zeros(T, H, D, dtype=BF, device=DEV)
    n = [T - 200, 200]
    g = torch.Generator().manual_seed(10)
    tail = [torch.randn(200, 2, D, generator=g).to(BF) for _ in range(3)]
    k[-200:, -1] = tail[1][:, 0].to(DEV)
    q = torch.zeros(T, 2, D, dtype=BF, device=DEV)
    q[-200:] = tail[0].to(DEV)
    cu_q, cu_k = offsets([0, 200], DEV), offsets(n, DEV)
    out = sd.attn_prompt(q[-200:, :1], k[:, -1:], k[:, -1:], cu_q, cu_k)
    check(out, None, packed_reference(tail[0][:, :1], tail[1][:, :1], tail[1][:, :1], [200], [200], 1), BF)


def test_repeated_call_is_the_same_to_the_bit_and_other_streams():
    g = torch.Generator().manual_seed(11)
    n = [300, 77, 500]
    q, k, v = (torch.randn(sum(n), h, 128, generator=g).to(BF).to(DEV) for h in (8, 2, 2))
    cu = offsets(n, DEV)
    a = sd.attn_prompt(q, k, v, cu)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = sd.attn_prompt(q, k, v, cu, stream=s)
    with torch.cuda.stream(s):
        c = sd.attn_prompt(q, k, v, cu)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("dtype,H", [(BF, 4), (BF, 32), (BF, 256), (F32, 4), (F32, 32)])
def test_replayed_from_a_graph(dtype, H):
    """The offsets are read when the kernel runs: a captured call serves other divisions of the same tokens."""
    T, D = 1000, 128
    g = torch.Generator().manual_seed(12)
    q, k, v = (torch.empty(T, H, D, dtype=dtype, device=DEV) for _ in range(3))
    cu, out, lse = offsets([300, 700, 0], DEV), torch.empty_like(q), torch.empty(H, T, device=DEV)
    side = torch.cuda.Stream()
    for t in (q, k, v):
        t.normal_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sd.attn_prompt(q, k, v, cu, out=out, lse_out=lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.attn_prompt(q, k, v, cu, out=out, lse_out=lse)
    for n in ([300, 700, 0], [1, 499, 500], [0, 0, 1000], [40, 256, 128]):
        for t in (q, k, v):
            t.copy_(_rows(T, H, D, dtype, g))
        cu.copy_(offsets(n, DEV))
        out.fill_(3.0)
        lse.fill_(3.0)
        want, want_lse = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
        sd.attn_prompt(q, k, v, cu, out=want, lse_out=want_lse)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        assert (out[:sum(n)] != 3.0).any() and (out[sum(n):] == 3.0).all()


@pytest.mark.parametrize("mask_block", [1, 32, 100])
@pytest.mark.parametrize("dtype,D", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
def test_last_value_of_a_sequence_is_infinite(dtype, D, mask_block):
    """Only the rows that see it show it, and they show an infinity: nothing that lies behind it takes part."""
    n = [141, 77]

    def edit(q, k, v):
        v[140] = math.inf

    q, k, v, out, lse = _run(n, None, 2, 1, D, dtype, mask_block, seed=13, extra=3, edit=edit)
    clean = _run(n, None, 2, 1, D, dtype, mask_block, seed=13, extra=3)
    want = packed_reference(clean[0], clean[1], clean[2], n, n, mask_block)
    first = 140 // mask_block * mask_block
    for rows in (slice(0, first), slice(141, 218)):
        check(out[rows], lse[:, rows], tuple(w[:, rows] if i == 1 else w[rows] for i, w in enumerate(want)), dtype, f"rows {rows}")
    assert (out[first:141] == math.inf).all()


def test_any_large_block_hides_nothing():
    x = torch.randn(50, 2, 64, device=DEV).to(BF)
    cu = offsets([50], DEV)
    whole = sd.attn_prompt(x, x, x, cu, mask_block=50)
    for block in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 1, 2 ** 70):
        assert torch.equal(sd.attn_prompt(x, x, x, cu, mask_block=block), whole)
    with pytest.raises(sd.SparsedError):
        sd.attn_prompt(x, x, x, cu, mask_block=0)
