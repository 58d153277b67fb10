"""The forms of a prompt call by its size (bf16: 32, 128 and 256 rows a work-group; fp32: 16 and 32), each at the edges: a call of many heads takes the
form of a large one at lengths that are checked quickly. A few heads are compared with the formula in 64 bits."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import check, offsets, packed_reference

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32

# heads that bring calls of 770 tokens and more to each form: tokens x heads up to 16384 (32768 at head dim 64), tokens / 256 x heads
# from 512 on, and between; the forms with large tiles also want sequences of some length on average (_run sees to that)
FORMS = [("few", BF, 128, 6, 2), ("few", BF, 64, 8, 8), ("128", BF, 128, 28, 4), ("128", BF, 64, 56, 28), ("256", BF, 128, 176, 22),
         ("256", BF, 64, 12, 4), ("few", F32, 128, 6, 2), ("few", F32, 64, 8, 8), ("32", F32, 128, 28, 4), ("32", F32, 64, 56, 28)]


def _average(form, D):
    """Tokens of a sequence from which on a call takes the form."""
    return {"few": 0, "256": 256 if D == 128 else 4096}.get(form, 9)


def _run(form, n_q, n_k, dtype, D, Hq, Hkv, mask_block, seed, edit=None, extra=2):
    print(f"prompt {n_q} over {n_k}, heads {Hq}/{Hkv} of {D}, {dtype}, blocks of {mask_block}", flush=True)
    g = torch.Generator().manual_seed(seed)
    more = _average(form, D) * (len(n_q) + 1) - sum(n_q)
    if more > 0:                          # a longer sequence behind them, which brings the average up
        same = n_q is n_k
        n_q, n_k = n_q + [more], n_k + [more]
        n_k = n_q if same else n_k
    T, Tk = sum(n_q), sum(n_k)
    q = torch.randn(T + extra, Hq, D, generator=g).to(dtype)
    k, v = (torch.randn(Tk + extra, Hkv, D, generator=g).to(dtype) for _ in range(2))
    if edit is not None:
        edit(q, k, v)
    out = torch.full((T + extra, Hq, D), 7.0, dtype=dtype, device=DEV)
    lse = torch.full((Hq, T + extra), 7.0, device=DEV)
    cu_k = offsets(n_k, DEV) if n_k is not n_q else None
    sd.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), offsets(n_q, DEV), cu_k, mask_block=mask_block, out=out, lse_out=lse)
    torch.cuda.synchronize()
    assert (out[T:] == 7.0).all() and (lse[:, T:] == 7.0).all()
    return q, k, v, out, lse


def _check_heads(q, k, v, out, lse, n_q, n_k, mask_block, rows=None, what=""):
    Hq, group = q.shape[1], q.shape[1] // k.shape[1]
    for h in sorted({0, Hq // 2 + 1, Hq - 1}):
        hk = h // group
        want = packed_reference(q[:, h:h + 1], k[:, hk:hk + 1], v[:, hk:hk + 1], n_q, n_k, mask_block)
        T = sum(n_q)
        got, gl = out[:T, h:h + 1], lse[h:h + 1, :T]
        if rows is not None:
            got, gl = got[rows], gl[:, rows]
            want = tuple(w[:, rows] if i == 1 else w[rows] for i, w in enumerate(want))
        check(got, gl, want, q.dtype, f"{what} head {h}")


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("mask_block", [1, 32, 7, 1 << 30])
def test_ragged_batch(form, dtype, D, Hq, Hkv, mask_block):
    n = [1, 300, 0, 129, 257, 64, 33]
    q, k, v, out, lse = _run(form, n, n, dtype, D, Hq, Hkv, mask_block, 1)
    _check_heads(q, k, v, out, lse, n, n, mask_block, what=form)


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", [f for f in FORMS if f[0] != "256"] + [("256", BF, 128, 8, 2)])
def test_one_long_and_many_short(form, dtype, D, Hq, Hkv):
    """More sequences than a wave has lanes; the tiles of the long one come first in the order."""
    n = [3] * 40 + [520] + [1, 0] * 30 + [100]
    q, k, v, out, lse = _run(form, n, n, dtype, D, Hq, Hkv, 1, 2)
    _check_heads(q, k, v, out, lse, n, n, 1, what=form)


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv,n", [("few", BF, 128, 4, 2, 5), ("few", F32, 64, 8, 2, 5), ("128", BF, 128, 4, 2, 25),
                                                   ("128", BF, 64, 3, 3, 25), ("256", BF, 128, 4, 2, 270), ("32", F32, 128, 4, 4, 25)])
def test_hundreds_of_sequences(form, dtype, D, Hq, Hkv, n):
    lens = [1 + (i * 37) % (2 * n) for i in range(600)]
    lens[2], lens[300], lens[555], lens[570:580] = 700, 0, 513, [0] * 10
    first = [sum(lens[:i]) for i in range(601)]
    q, k, v, out, lse = _run(form, lens, lens, dtype, D, Hq, Hkv, 1, 9)
    for s in (0, 2, 3, 63, 64, 299, 301, 511, 512, 555, 580, 599):
        a, e = first[s], first[s + 1]
        _check_heads(q[a:e], k[a:e], v[a:e], out[a:e], lse[:, a:e], [e - a], [e - a], 1, what=f"{form} {s}")


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("n_q,n_k", [([700, 70], [1000, 200]), ([400, 300, 80], [370, 0, 81]), ([768], [64]), ([1] * 3 + [767], [5, 1, 0, 800])], ids=str)
def test_other_key_lengths(form, dtype, D, Hq, Hkv, n_q, n_k):
    q, k, v, out, lse = _run(form, n_q, n_k, dtype, D, Hq, Hkv, 1, 3)
    _check_heads(q, k, v, out, lse, n_q, n_k, 1, what=form)


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan], ids=str)
def test_hidden_places_do_not_matter(form, dtype, D, Hq, Hkv, bad):
    n, cut = [90, 600, 100], 90 + 333

    def edit(q, k, v):
        k[cut], v[cut + 1] = bad, bad
        v[90 + 599] = bad                 # the last token of a sequence: hidden from all others of its tile
        k[-2:], v[-2:] = bad, bad

    q, k, v, out, lse = _run(form, n, n, dtype, D, Hq, Hkv, 1, 4, edit)
    clean = _run(form, n, n, dtype, D, Hq, Hkv, 1, 4)
    for rows in (slice(0, cut), slice(690, 790)):
        _check_heads(*clean[:3], out, lse, n, n, 1, rows, f"{form} {bad}")
    assert not torch.isfinite(out[cut + 1:690]).any()


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("mask_block", [1, 32])
def test_last_value_of_a_sequence_is_infinite(form, dtype, D, Hq, Hkv, mask_block):
    """Only the rows that see it show it."""
    n = [700, 77]

    def edit(q, k, v):
        v[699] = math.inf

    q, k, v, out, lse = _run(form, n, n, dtype, D, Hq, Hkv, mask_block, 5, edit)
    clean = _run(form, n, n, dtype, D, Hq, Hkv, mask_block, 5)
    first = 699 // mask_block * mask_block
    for rows in (slice(0, first), slice(700, 777)):
        _check_heads(*clean[:3], out, lse, n, n, mask_block, rows, form)
    assert (out[first:700] == math.inf).all()


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("sign", [1, -1])
def test_logits_that_climb_or_fall(form, dtype, D, Hq, Hkv, sign):
    n = [650, 130]

    def edit(q, k, v):
        q[:, :, 0] = 8.0
        k[:, :, 0] = (sign * torch.arange(k.shape[0]).float() * (0.125 * D ** 0.5))[:, None].to(dtype)

    q, k, v, out, lse = _run(form, n, n, dtype, D, Hq, Hkv, 1, 6, edit)
    _check_heads(q, k, v, out, lse, n, n, 1, what=form)


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
def test_strided_views_and_repeats(form, dtype, D, Hq, Hkv):
    g = torch.Generator().manual_seed(7)
    n = [500, 283, max(0, 3 * _average(form, D) - 783)]
    T = sum(n)
    qkv = torch.randn(T, Hq + 2 * Hkv, D, generator=g).to(dtype)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    dev = qkv.to(DEV)
    args = dev[:, :Hq], dev[:, Hq:Hq + Hkv], dev[:, Hq + Hkv:], offsets(n, DEV)
    out = torch.full((Hq, T, D), 5.0, dtype=dtype, device=DEV)
    lse = torch.empty(Hq, T, device=DEV)
    sd.attn_prompt(*args, out=out.transpose(0, 1), lse_out=lse)
    _check_heads(q, k, v, out.transpose(0, 1), lse, n[:2], n[:2], 1, what=form)
    again = sd.attn_prompt(*args)
    torch.cuda.synchronize()
    assert torch.equal(again, out.transpose(0, 1))


@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
def test_offsets_out_of_range_stay_inside(form, dtype, D, Hq, Hkv):
    """Offsets that descend, leave the array or name rows twice."""
    g = torch.Generator().manual_seed(8)
    T = max(800, 5 * _average(form, D) + 20)
    q = torch.randn(T, Hq, D, generator=g).to(dtype).to(DEV)
    k, v = (torch.randn(T, Hkv, D, generator=g).to(dtype).to(DEV) for _ in range(2))
    for cu in ([0, 300, 5000, -7], [0, T, 0, T, 0, T], [-100, 2 ** 31 - 1], [T, 0]):
        out = torch.full((T, Hq, D), 9.0, dtype=dtype, device=DEV)
        sd.attn_prompt(q, k, v, torch.tensor(cu, dtype=torch.int32, device=DEV), out=out)
        torch.cuda.synchronize()
        assert torch.isfinite(out).all()
    assert (out == 9.0).all()
