"""Timed cases of attention with a paged key/value cache: what a program calls that generates block by block (or token by
token) and keeps the keys and values of what is finished, from one token of one sequence to long prompts.

Three operators, reached through the package's entry points:

  append   ``cache_append``: keys and values of new tokens, packed, into the pages of their sequences
  prompt   ``attn_prompt``: attention over whole prompts, packed one behind the other, with grouped heads; a token sees the
           tokens up to the end of its own block of ``mask_block`` tokens (1: causal)
  paged    ``attn_paged``: attention of the last tokens of every sequence (one, or a block) over its pages

A case is a plain dict. ``own`` chooses between the package's calls and the same operators in elementary torch operations.
Head shapes are those of ``workload/configs.py``; lengths and page sizes are generic.
"""
import math
import random

import torch

own = False
DEVICE = "cuda"


def listed():
    return [
        # one token each of a few short sequences: the latency of the smallest call
        _case("append_token_8", "append", "bf16", 8, 2, 2, 64, 20, 256, page=16, new=1),
        # the keys and values of a batch of prompts, once they are computed
        _case("append_prompts", "append", "bf16", 8, 32, 32, 128, 1000, 16384, page=64, new=0),
        # many short prompts of a small layer, packed: ragged, far from filling tiles
        _case("prompt_short_d64", "prompt", "bf16", 24, 8, 2, 64, 1, 600),
        # one prompt of the 4k workload
        _case("prompt_4k", "prompt", "bf16", 1, 32, 32, 128, 4096, 4096),
        # a batch of prompts of a grouped-query layer, log-sum-exp kept
        _case("prompt_packed_gqa", "prompt", "bf16", 6, 28, 4, 128, 200, 6000, lse=True),
        # prompts of a model that attends within blocks of 32 tokens in both directions
        _case("prompt_blocks32", "prompt", "bf16", 3, 32, 32, 128, 700, 3000, mask_block=32),
        # the longest prompt: grouped heads at 32k, the largest pass
        _case("prompt_32k_gqa", "prompt", "bf16", 1, 28, 4, 128, 32768, 32768),
        # fp32 at an ordinary size, log-sum-exp kept
        _case("prompt_2000_f32", "prompt", "f32", 2, 8, 8, 128, 300, 2000, lse=True),
        # one token of one short sequence, fp32: the latency of the smallest attention call
        _case("paged_token_f32", "paged", "f32", 1, 2, 2, 64, 256, 256, page=16, new=1),
        # a serving batch: one token each of 32 sequences of very different length, small pages
        _case("paged_batch_32", "paged", "bf16", 32, 32, 32, 128, 500, 8000, page=16, new=1),
        # one token of one long context, grouped heads: few rows, a long axis; pages hold one head after the other
        _case("paged_token_64k_gqa", "paged", "bf16", 1, 28, 4, 128, 65536, 65536, page=64, new=1, heads_first=True),
        # a block of 32 new tokens, seen in both directions, at the end of each of four sequences
        _case("paged_blocks32", "paged", "bf16", 4, 32, 32, 128, 1000, 8000, page=32, new=32, mask_block=32),
    ]


def _case(name, op, dtype, n_seqs, Hq, Hkv, D, lo, hi, page=0, new=0, mask_block=1, lse=False, heads_first=False, salt=0):
    c = dict(op=op, dtype=dtype, n_seqs=n_seqs, Hq=Hq, Hkv=Hkv, D=D, lo=lo, hi=hi, page=page, new=new, mask_block=mask_block,
             lse=lse, heads_first=heads_first, salt=salt)
    return dict(name=name, **c) if name else c


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: operator, heads, lengths (spread over their logarithm, mostly odd), pages and blocks of the same ranges."""
    op = rng.choice(["append", "prompt", "prompt", "prompt", "paged", "paged", "paged"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    D = rng.choice([64, 128, 128])
    Hq, Hkv = rng.choice([(2, 2), (8, 2), (8, 8), (28, 4), (32, 32)])
    block = rng.choice([1, 1, 1, 4, 32])
    lse, heads_first, salt = rng.random() < 0.3, rng.random() < 0.4, rng.randrange(1 << 20)
    if op == "prompt":
        hi = _log_uniform(rng, 16, 3000 if dtype == "f32" else 16384)
        n = _log_uniform(rng, 1, max(1, min(24, 32768 // hi)))
        return _case("", op, dtype, n, Hq, Hkv, D, max(1, _log_uniform(rng, 1, hi)), hi, mask_block=block, lse=lse, salt=salt)
    page = rng.choice([16, 32, 64, 128])
    hi = _log_uniform(rng, 16, 65536 if Hkv < 32 else 16384)
    n = _log_uniform(rng, 1, max(1, min(48, (200000 if Hkv < 32 else 60000) // hi)))
    if dtype == "f32":
        n = (n + 1) // 2
    lo = _log_uniform(rng, 1, hi)
    if op == "append":
        return _case("", op, dtype, n, Hkv, Hkv, D, lo, hi, page=page, new=rng.choice([0, 1, 32]), heads_first=heads_first, salt=salt)
    new = rng.choice([1, 1, 1, 5, 32])
    return _case("", op, dtype, n, Hq, Hkv, D, lo, hi, page=page, new=new, mask_block=block, lse=lse, heads_first=heads_first, salt=salt)


def _lengths(case):
    """Tokens of every sequence: the first has the most, the others spread over the range."""
    rng = random.Random(case["salt"])
    return [case["hi"]] + [_log_uniform(rng, case["lo"], case["hi"]) for _ in range(case["n_seqs"] - 1)]


def _new_tokens(case, lens):
    """How many of them are the call's: all of a prompt, else the last few, fewer in some sequences."""
    if case["new"] == 0:
        return list(lens)
    rng = random.Random(case["salt"] + 1)
    most = case["new"]
    return [min(n, most if s % 2 == 0 else rng.randint(1, most)) for s, n in enumerate(lens)]


# ------------------------------------------------------------------------------------------------ inputs


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dt, D, Hq, Hkv = _dtype(case), case["D"], case["Hq"], case["Hkv"]
    lens = _lengths(case)
    new = _new_tokens(case, lens)
    T = sum(new)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=dt)

    s = dict(op=case["op"], lens=lens, new=new, mask_block=case["mask_block"])
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    # one token each needs no offsets
    s["cu"] = torch.tensor(cu, dtype=torch.int32, device=DEVICE) if max(new) > 1 else None
    # a direction that the queries share and the first tokens answer: trained models put weight on the first tokens
    sink = torch.randn(D, generator=gen, device=DEVICE, dtype=torch.float32)
    sink = sink * (4.0 / sink.norm())
    if case["op"] != "append":
        s["q"] = normal(T, Hq, D) + sink.to(dt)
        s["out"] = torch.zeros(T, Hq, D, dtype=dt, device=DEVICE)
        s["lse"] = torch.zeros(Hq, T, dtype=torch.float32, device=DEVICE) if case["lse"] else None
    if case["op"] != "paged":
        s["k"], s["v"] = normal(T, Hkv, D), normal(T, Hkv, D)
    if case["op"] == "prompt":
        for at in cu[:-1]:
            s["k"][at] += (3.0 * sink).to(dt)
        return s
    ps = case["page"]
    counts = [-(-n // ps) for n in lens]
    n_pages = sum(counts) + 3
    shape = (n_pages, Hkv, ps, D) if case["heads_first"] else (n_pages, ps, Hkv, D)
    s["cache_k"], s["cache_v"] = (normal(*shape) for _ in range(2))
    if case["heads_first"]:
        s["cache_k"], s["cache_v"] = s["cache_k"].transpose(1, 2), s["cache_v"].transpose(1, 2)
    free = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.zeros(len(lens), max(counts) + 1, dtype=torch.int32)
    for b, n in enumerate(counts):
        for t in range(n):
            table[b, t] = free.pop()
    s["table"] = table.to(DEVICE)
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    if case["op"] == "paged":
        s["cache_k"][table[:, 0].long().to(DEVICE), 0] += (3.0 * sink).to(dt)
    return s


# ------------------------------------------------------------------------------------------------ one pass


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2509_24014_amd as sd

    if s["op"] == "prompt":
        out = sd.attn_prompt(s["q"], s["k"], s["v"], s["cu"], mask_block=s["mask_block"], out=s["out"], lse_out=s["lse"])
        return out if s["lse"] is None else (out, s["lse"])
    if "cache" not in s:   # the handle that a program keeps, and the scratch memory beside it
        s["cache"] = sd.PagedCache(s["cache_k"], s["cache_v"], s["table"], s["seq_lens"])
        if s["op"] == "paged":
            s["workspace"] = torch.empty(sd.paged_workspace_bytes(s["q"], s["cache"]), dtype=torch.uint8, device=DEVICE)
    if s["op"] == "append":
        sd.cache_append(s["cache"], s["k"], s["v"], s["cu"])
        return s["cache_k"], s["cache_v"]
    out = sd.attn_paged(s["q"], s["cache"], s["cu"], mask_block=s["mask_block"], out=s["out"], lse_out=s["lse"],
                        workspace=s["workspace"])
    return out if s["lse"] is None else (out, s["lse"])


def _run_plain(s):
    if s["op"] == "append":
        return _plain_append(s)
    out, lse = s["out"], s["lse"]
    at = 0
    for b, n in enumerate(s["new"]):
        q = s["q"][at:at + n].float()
        if s["op"] == "prompt":
            k, v = s["k"][at:at + n].float(), s["v"][at:at + n].float()
        else:
            m = s["lens"][b]
            ps = s["cache_k"].shape[1]
            pages = s["table"][b, :-(-m // ps)].long()
            k, v = (c[pages].flatten(0, 1)[:m].float() for c in (s["cache_k"], s["cache_v"]))
        _plain_attention(q, k, v, s["mask_block"], out[at:at + n], None if lse is None else lse[:, at:at + n])
        at += n
    return out if lse is None else (out, lse)


def _plain_attention(q, k, v, mask_block, out, lse):
    """The last n of a sequence's m tokens over its keys, some rows and heads at a time."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[0], k.shape[1]
    group = Hq // Hkv
    qh = q.transpose(0, 1).reshape(Hkv, group, n, D)
    kt, vh = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
    rows = max(1, min(n, (1 << 28) // (Hq * m)))
    scale = 1.0 / math.sqrt(D)
    for r in range(0, n, rows):
        e = min(n, r + rows)
        last = m - n + torch.arange(r, e, device=q.device)                      # where the token stands in its sequence
        seen = (last // mask_block + 1) * mask_block
        far = min(m, ((m - n + e - 1) // mask_block + 1) * mask_block)          # no row of these sees past here
        qs = qh[:, :, r:e].reshape(Hkv, group * (e - r), D) * scale
        s = torch.matmul(qs, kt[:, :, :far]).view(Hkv, group, e - r, far)
        s = s.masked_fill(torch.arange(far, device=q.device) >= seen[:, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        p = (s - top).exp()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(Hkv, group * (e - r), far), vh[:, :far]).view(Hkv, group, e - r, D) / total
        out[r:e] = o.view(Hq, e - r, D).transpose(0, 1).to(out.dtype)
        if lse is not None:
            lse[:, r:e] = (top + total.log()).view(Hq, e - r)


def _plain_append(s):
    new = torch.tensor(s["new"], device=DEVICE)
    T, ps = s["k"].shape[0], s["cache_k"].shape[1]
    first = torch.cumsum(new, 0) - new
    b = torch.repeat_interleave(torch.arange(len(s["new"]), device=DEVICE), new, output_size=T)
    at = s["seq_lens"].long()[b] - new[b] + torch.arange(T, device=DEVICE) - first[b]
    page, slot = s["table"].long()[b, at // ps], at % ps
    s["cache_k"][page, slot] = s["k"]
    s["cache_v"][page, slot] = s["v"]
    return s["cache_k"], s["cache_v"]


# ------------------------------------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        k, v = s["cache_k"].clone(), s["cache_v"].clone()
        table, ps, at = s["table"].tolist(), case["page"], 0
        for b, (m, n) in enumerate(zip(s["lens"], s["new"])):
            first = m - n
            while first < m:     # a run of tokens in one page
                run_end = min(m, (first // ps + 1) * ps)
                page, slot, count = table[b][first // ps], first % ps, run_end - first
                k[page, slot:slot + count] = s["k"][at:at + count]
                v[page, slot:slot + count] = s["v"][at:at + count]
                at, first = at + count, run_end
        return k, v
    Hq, group, D, mb = case["Hq"], case["Hq"] // case["Hkv"], case["D"], case["mask_block"]
    T = sum(s["new"])
    out = torch.zeros(T, Hq, D, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(Hq, T, dtype=torch.float64, device=DEVICE)
    at = 0
    for b, (m, n) in enumerate(zip(s["lens"], s["new"])):
        if case["op"] == "prompt":
            keys, values = s["k"][at:at + n], s["v"][at:at + n]
        else:
            token = torch.arange(m, device=DEVICE)
            page, slot = s["table"][b].long()[token // case["page"]], token % case["page"]
            keys, values = s["cache_k"][page, slot], s["cache_v"][page, slot]
        for h in range(Hq):
            kd, vd = keys[:, h // group].double(), values[:, h // group].double()
            for r in range(0, n, 4096):
                e = min(n, r + 4096)
                logits = s["q"][at + r:at + e, h].double() @ kd.T.contiguous() / math.sqrt(D)
                i = torch.arange(m - n + r, m - n + e, device=DEVICE)[:, None]
                j = torch.arange(m, device=DEVICE)[None, :]
                logits[j // mb > i // mb] = -math.inf        # a token of a later block is not seen
                norm = torch.logsumexp(logits, 1)
                out[at + r:at + e, h] = torch.exp(logits - norm[:, None]) @ vd
                lse[h, at + r:at + e] = norm
        at += n
    return (out, lse) if case["lse"] else out


# ------------------------------------------------------------------------------------------------ accounting


def work(case):
    """Inputs read once, outputs written once; both matrix products over the pairs that are seen."""
    el = 2 if case["dtype"] == "bf16" else 4
    Hq, Hkv, D, mb = case["Hq"], case["Hkv"], case["D"], case["mask_block"]
    lens = _lengths(case)
    new = _new_tokens(case, lens)
    T = sum(new)
    if case["op"] == "append":
        return {"bytes": 4 * T * Hkv * D * el, "flops": 0}
    pairs = 0
    for m, n in zip(lens, new):
        pairs += sum(min(m, (i // mb + 1) * mb) for i in range(m - n, m))
    keys = T if case["op"] == "prompt" else sum(lens)
    table = 0 if case["op"] == "prompt" else 4 * sum(-(-m // case["page"]) for m in lens)
    return {"bytes": (2 * T * Hq + 2 * keys * Hkv) * D * el + table + (4 * T * Hq if case["lse"] else 0),
            "flops": 4.0 * Hq * D * pairs}
