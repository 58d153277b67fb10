"""Helpers of the tests of attention with a paged cache (not a test module): the formulas in 64 bits on the CPU, and how far a
result in fp32 or bf16 may be from them.

Bounds, per output element, with A = sum p |v| / sum p, half steps u = 2^-24 (fp32) and 2^-8 (bf16):
  logits      a sum of D products, each rounded, in fp32: D u_32 sum |q k| / sqrt(D), and its scaling: a few u_32 |s|
  exponent    s c - M in fp32: u_32 (|s c| + |M|), and 2^x itself to 2 u_32; a p is off by that much of itself, and so is
              their sum: twice
  sums        n terms in fp32: n u_32
  bf16        p rounded before the product with V: 2^-8 A, and the result rounded: 2^-8 |o|
  joining     of parts, a factor each: a few u_32
"""
import math

import torch

U32, UBF = 2.0 ** -24, 2.0 ** -8


def seen(p, m, mask_block):
    return 0 if p < 0 else min(m, (p // mask_block + 1) * mask_block)


def attend64(q, k, v, mask_block):
    """q [n, Hq, D], k, v [m, Hkv, D]: out [n, Hq, D], lse [Hq, n], and the two scales of the bounds: A [n, Hq, D] and
    per row the error of a p relative to itself [n, Hq]."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[0], k.shape[1]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    out, A = torch.zeros(n, Hq, D, dtype=torch.float64), torch.zeros(n, Hq, D, dtype=torch.float64)
    lse, rel = torch.full((Hq, n), -math.inf, dtype=torch.float64), torch.zeros(n, Hq, dtype=torch.float64)
    for i in range(n):
        far = seen(m - n + i, m, mask_block)
        if far == 0:
            continue
        kk = k[:far].repeat_interleave(Hq // Hkv, 1).transpose(0, 1)     # [Hq, far, D]
        vv = v[:far].repeat_interleave(Hq // Hkv, 1).transpose(0, 1)
        s = (kk @ q[i][:, :, None])[..., 0] / math.sqrt(D)
        top = s.amax(1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(1, keepdim=True)
        lse[:, i] = (top + total.log())[:, 0]
        out[i] = (p[:, None, :] @ vv)[:, 0] / total
        A[i] = (p[:, None, :] @ vv.abs())[:, 0] / total
        products = (kk.abs() @ q[i].abs()[:, :, None])[..., 0] / math.sqrt(D)
        rel[i] = U32 * (D * products + 12 * s.abs() + 8).amax(1) + far * U32
    return out, lse, A, rel


def check(got, got_lse, want, dtype, what=""):
    out, lse, A, rel = want
    g = got.detach().double().cpu()
    bound = A * (2.0 * rel[..., None]) + 8 * U32 * A
    if dtype == torch.bfloat16:
        bound += UBF * A + UBF * out.abs()
    else:
        bound += U32 * out.abs()
    bound += 2.0 ** -126
    assert torch.isfinite(g).all(), f"{what}: not finite"
    over = (g - out).abs() - bound
    assert (over <= 0).all(), f"{what}: off by {(g - out).abs().max():.3e}, {(over > 0).sum()} elements beyond their bound (up to {over.max():.3e} over)"
    if got_lse is not None:
        gl = got_lse.detach().double().cpu()
        empty = torch.isinf(lse)
        assert (gl[empty] == -math.inf).all(), f"{what}: rows that see nothing"
        lb = rel.T + 2 * U32 * lse.abs().nan_to_num(posinf=0.0) + 4 * U32
        d = (gl - lse).abs()[~empty]
        assert (d <= lb[~empty]).all(), f"{what}: log-sum-exp off by {d.max():.3e}"


def offsets(counts, device="cpu"):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, dtype=torch.int32, device=device)


def packed_reference(q, k, v, n_q, n_k, mask_block):
    """attend64 over every sequence, one behind the other."""
    parts, at_q, at_k = [], 0, 0
    for a, b in zip(n_q, n_k):
        parts.append(attend64(q[at_q:at_q + a], k[at_k:at_k + b], v[at_k:at_k + b], mask_block))
        at_q, at_k = at_q + a, at_k + b
    return tuple(torch.cat([p[i] for p in parts], 1 if i == 1 else 0) for i in range(4))


def make_cache(lens, Hkv, D, dtype, page, seed, heads_first=False, spare=2, fill=float("nan"), device="cuda:0", room=1):
    """Pages in a random order, keys and values of lens tokens in them; every other place holds `fill`. Returns
    (k_pages, v_pages, page_table, seq_lens) on the device and the lists of keys and values per sequence on the CPU."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + spare
    shape = (n_pages, Hkv, page, D) if heads_first else (n_pages, page, Hkv, D)
    pages = [torch.full(shape, fill, dtype=dtype) for _ in range(2)]
    views = [p.transpose(1, 2) if heads_first else p for p in pages]
    free = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((len(lens), max(counts + [0]) + room), -5, dtype=torch.int32)
    rows = []
    for s, n in enumerate(lens):
        kv = [torch.randn(n, Hkv, D, generator=g).to(dtype) for _ in range(2)]
        rows.append(kv)
        for t in range(counts[s]):
            table[s, t] = free.pop()
            count = min(page, n - t * page)
            for view, x in zip(views, kv):
                view[table[s, t], :count] = x[t * page:t * page + count]
    dev = [p.to(device) for p in pages]
    dev = [p.transpose(1, 2) if heads_first else p for p in dev]
    return dev[0], dev[1], table.to(device), torch.tensor(lens, dtype=torch.int32, device=device), rows


def paged_reference(q, rows, new, mask_block):
    parts, at = [], 0
    for (k, v), n in zip(rows, new):
        parts.append(attend64(q[at:at + n], k, v, mask_block))
        at += n
    return tuple(torch.cat([p[i] for p in parts], 1 if i == 1 else 0) for i in range(4))
