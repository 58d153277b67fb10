"""Prompt attention where logits are finite and very large or very small: every form gives what the softmax of them is. One column of
queries and keys holds the logits, so that equal keys have equal ones and the values' mean is the result."""
import math

import pytest
import torch

import paper_2509_24014_amd as sd
from cache_utils import U32, UBF, offsets
from test_gpu_prompt_forms import FORMS, _average

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
A0, B0 = 1 + 11 / 128, 1 + 23 / 128    # eight bits each, as bf16 has them: the product of such a logit with the scale of the exponent is rounded in fp32


def _means(form, dtype, D, Hq, Hkv, q0, k0, n=400):
    """Causal attention of one sequence (a longer one behind it where the form wants that); k0: the keys' column. Rows of the first sequence:
    out and lse, and from the definition the mean of |v| over the keys with the largest logit, that of v, and the log-sum-exp."""
    more = max(0, max(_average(form, D), 385) * 2 - n)
    T = n + more
    g = torch.Generator().manual_seed(40)
    q, k = torch.zeros(T, Hq, D, dtype=dtype), torch.zeros(T, Hkv, D, dtype=dtype)
    v = torch.randn(T, Hkv, D, generator=g).to(dtype)
    q[:, :, 0], k[:n, :, 0] = q0, k0[:n, None].to(dtype)
    lse = torch.empty(Hq, T, device=DEV)
    out = sd.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), offsets([n, more], DEV), lse_out=lse)
    torch.cuda.synchronize()
    logits = (q[:n, 0, 0].double()[:, None] * k[:n, 0, 0].double()) / math.sqrt(D)
    logits[torch.ones(n, n).triu(1).bool()] = -math.inf
    w = torch.softmax(logits, 1)
    h = (0, Hq // 2 + 1, Hq - 1)
    vd = v[:n, [x // (Hq // Hkv) for x in h]].double()
    return out[:n, h].double().cpu(), lse[h, :n].double().cpu(), torch.einsum("ij,jhd->ihd", w, vd.abs()), torch.einsum("ij,jhd->ihd", w, vd), torch.logsumexp(logits, 1)


# Weights are equal and results means of up to 400 values: P rounded and the result rounded in bf16, each by half a step; the sum of n terms in
# fp32 n U32 of the mean of |v|; the exponents of equal logits are the same number, so a weight's own error, 4 U32, is all there is beside them.
@pytest.mark.parametrize("form,dtype,D,Hq,Hkv", FORMS)
@pytest.mark.parametrize("q0,k0", [(2.0 ** 60, -2.0 ** 60), (2.0 ** 60, 2.0 ** 60), (2.0 ** 20, -2.0 ** 16), (2.0 ** 20, 2.0 ** 16), (2.0 ** 17, -2.0 ** 15),
                                   (2.0 ** 16, 2.0 ** 12), (2.0 ** 16, -2.0 ** 15), (A0 * 2.0 ** 60, -B0 * 2.0 ** 60), (A0 * 2.0 ** 60, B0 * 2.0 ** 60),
                                   (A0 * 2.0 ** 20, -B0 * 2.0 ** 18), (A0 * 2.0 ** 20, B0 * 2.0 ** 18), (A0 * 2.0 ** 17, -B0 * 2.0 ** 16),
                                   (A0 * 2.0 ** 17, B0 * 2.0 ** 16), (A0 * 2.0 ** 16, -B0 * 2.0 ** 14), (A0 * 2.0 ** 16, B0 * 2.0 ** 14)], ids=str)
@pytest.mark.parametrize("first", [0, 45], ids=["equal", "switch"])
def test_equal_logits_of_any_size(form, dtype, D, Hq, Hkv, q0, k0, first):
    """`switch`: the keys from the 45th on have logits of 0, so that rows behind it leave a range (k0 < 0) or stay in it (k0 > 0)."""
    print(f"{form} {dtype} {D} {Hq}/{Hkv}, {q0} x {k0}, {first}", flush=True)
    column = torch.full((400,), k0)
    if first:
        column[first:] = 0.0
    out, lse, A, want, want_lse = _means(form, dtype, D, Hq, Hkv, q0, column)
    step = UBF if dtype == BF else U32
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert ((out - want).abs() <= (2 * step + (400 + 8) * U32) * A).all(), (out - want).abs().max()
    assert ((lse - want_lse).abs() <= 8 * U32 * want_lse.abs() + (400 + 8) * U32).all()
