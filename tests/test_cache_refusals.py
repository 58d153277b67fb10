"""What the entry points with a key/value cache refuse, and the layout of their structs. Nothing here launches a kernel: every call
fails validation on the host (the fake device pointers are never touched) or has nothing to do."""
import ctypes

import pytest
import torch

from paper_2509_24014_amd import binding

R = ctypes.byref
BF, F32 = binding.SPARSED_BF16, binding.SPARSED_F32
NULL, SHAPE, DTYPE, STRIDE, RANGE, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5, 6, 7


def _packed(T=100, H=4, D=128, dtype=BF, data=0x1000, sl=None, sh=None, B=1):
    return binding._Tensor(data, dtype, B, H, T, D, 0, D if sh is None else sh, H * D if sl is None else sl)


def _pages(n=50, H=2, page=16, D=128, dtype=BF, data=0x2000, sb=None, sh=None, sl=None):
    sl = H * D if sl is None else sl
    return binding._Tensor(data, dtype, n, H, page, D, page * sl if sb is None else sb, D if sh is None else sh, sl)


def _cache(k=None, v=None, table=0x3000, lens=0x4000, n_seqs=3, max_pages=8, stride=8):
    return binding._PagedCache(k or _pages(), v or _pages(), table, lens, n_seqs, max_pages, stride)


def _ex(ws=0x10000, size=1 << 40):
    return binding._Exec(None, ws, size, None, None, None, None)


CU = 0x5000


def test_prompt_refusals():
    f = binding.load_library().sparsed_attn_prompt
    q, kv = _packed(), _packed(H=2)

    def call(q=q, k=kv, v=kv, o=q, cu_q=CU, cu_k=None, n=3, block=1):
        return f(R(q), R(k), R(v), R(o), cu_q, cu_k, n, block, None)

    assert f(None, R(kv), R(kv), R(q), CU, None, 3, 1, None) == NULL
    assert call(q=_packed(data=None)) == NULL and call(o=_packed(data=None)) == NULL and call(cu_q=None) == NULL
    assert call(block=0) == RANGE and call(block=-5) == RANGE and call(n=-1) == RANGE
    assert call(q=_packed(D=96)) == UNSUPPORTED and call(q=_packed(T=(1 << 30) + 1)) == UNSUPPORTED
    assert call(q=_packed(dtype=7)) == DTYPE and call(k=_packed(H=2, dtype=F32)) == DTYPE and call(o=_packed(dtype=F32)) == DTYPE
    assert call(v=_packed(H=2, dtype=F32)) == DTYPE
    assert call(k=_packed(H=3)) == SHAPE and call(v=_packed(H=4)) == SHAPE and call(o=_packed(T=99)) == SHAPE and call(o=_packed(H=2)) == SHAPE
    assert call(q=_packed(B=2)) == SHAPE and call(q=_packed(T=-1)) == SHAPE and call(q=_packed(H=0)) == SHAPE
    assert call(k=_packed(H=2, D=64)) == SHAPE
    assert call(k=_packed(T=90, H=2), v=_packed(T=90, H=2)) == SHAPE                      # other keys need cu_k
    assert call(v=_packed(T=90, H=2), cu_k=CU) == SHAPE
    assert call(q=_packed(data=0x1008)) == STRIDE and call(q=_packed(sl=516)) == STRIDE and call(q=_packed(sh=4)) == STRIDE
    assert call(k=_packed(H=2, sl=64)) == STRIDE and call(q=_packed(sh=-128)) == STRIDE
    assert call(q=_packed(sl=1 << 23)) == STRIDE                                          # 128 rows of 2^24 bytes
    assert call(k=_packed(H=2, dtype=F32, sl=258), q=_packed(dtype=F32), v=_packed(H=2, dtype=F32), o=_packed(dtype=F32)) == STRIDE
    assert call(o=_packed(sh=64)) == STRIDE and call(o=_packed(sh=0)) == STRIDE            # heads of out in one place
    many = {"q": _packed(T=1 << 25), "k": _packed(T=1 << 25, H=2), "v": _packed(T=1 << 25, H=2), "o": _packed(T=1 << 25)}
    assert call(n=(1 << 30) + 1) == UNSUPPORTED
    assert call(n=1 << 24, **many) == UNSUPPORTED                                         # more work-groups than a launch has
    many = {"q": _packed(T=1 << 29, dtype=F32), "k": _packed(T=1 << 29, H=2, dtype=F32), "v": _packed(T=1 << 29, H=2, dtype=F32), "o": _packed(T=1 << 29, dtype=F32)}
    assert call(n=1, **many) == UNSUPPORTED
    # nothing to do: no pointers needed
    assert call(q=_packed(T=0, data=None), k=_packed(T=0, H=2, data=None), v=_packed(T=0, H=2, data=None), o=_packed(T=0, data=None)) == 0
    assert call(n=0, cu_q=None) == 0


def test_paged_refusals():
    f = binding.load_library().sparsed_attn_paged
    q = _packed(T=3)

    def call(q=q, c=None, cu=None, block=1, o=None, ex=None):
        return f(R(q), R(c or _cache()), cu, block, R(o or q), R(ex or _ex()))

    assert f(None, R(_cache()), None, 1, R(q), None) == NULL and f(R(q), None, None, 1, R(q), None) == NULL
    assert f(R(q), R(_cache()), None, 1, None, None) == NULL
    assert call(c=_cache(table=None)) == NULL and call(c=_cache(lens=None)) == NULL and call(c=_cache(k=_pages(data=None))) == NULL
    assert call(cu=CU, c=_cache(n_seqs=(1 << 30) + 1)) == UNSUPPORTED
    assert call(block=0) == RANGE and call(c=_cache(n_seqs=-1)) == RANGE and call(c=_cache(max_pages=-1)) == RANGE
    assert call(c=_cache(k=_pages(page=24), v=_pages(page=24))) == UNSUPPORTED and call(c=_cache(k=_pages(page=512), v=_pages(page=512))) == UNSUPPORTED
    assert call(c=_cache(k=_pages(D=32), v=_pages(D=32))) == UNSUPPORTED
    assert call(c=_cache(max_pages=1 << 27, stride=1 << 27)) == UNSUPPORTED                 # 2^31 tokens
    assert call(c=_cache(v=_pages(page=32))) == SHAPE and call(c=_cache(v=_pages(n=49))) == SHAPE and call(c=_cache(v=_pages(H=4))) == SHAPE
    assert call(c=_cache(k=_pages(n=0), v=_pages(n=0))) == SHAPE
    assert call(c=_cache(v=_pages(dtype=F32))) == DTYPE and call(c=_cache(k=_pages(dtype=F32), v=_pages(dtype=F32))) == DTYPE
    assert call(q=_packed(T=3, H=3), o=_packed(T=3, H=3)) == SHAPE and call(q=_packed(T=3, D=64), o=_packed(T=3, D=64)) == SHAPE
    assert call(q=_packed(T=4)) == SHAPE and call(q=_packed(T=2)) == SHAPE                  # one token each, or offsets
    assert call(o=_packed(T=4)) == SHAPE
    assert call(c=_cache(stride=7)) == STRIDE
    assert call(c=_cache(k=_pages(sl=252))) == STRIDE and call(c=_cache(k=_pages(sb=4100))) == STRIDE and call(c=_cache(k=_pages(data=0x2004))) == STRIDE
    assert call(c=_cache(k=_pages(sl=1 << 27))) == STRIDE                                   # a page of 2^32 bytes
    assert f(R(q), R(_cache()), None, 1, R(q), None) == WORKSPACE
    assert call(ex=_ex(size=16)) == WORKSPACE and call(ex=_ex(ws=0x10010)) == WORKSPACE and call(ex=_ex(ws=None)) == WORKSPACE
    many = _packed(T=1 << 22)                                                               # a work-group a row to join them: 2^24
    assert call(q=many, o=many, cu=CU) == UNSUPPORTED
    assert call(o=_packed(T=3, sh=0)) == STRIDE
    empty = _packed(T=0, data=None)
    assert call(q=empty, o=empty, cu=CU) == 0
    none = _cache(n_seqs=0, table=None, lens=None)
    assert call(q=empty, o=empty, c=none) == 0 and call(c=none, cu=CU) == 0


def test_append_refusals():
    f = binding.load_library().sparsed_cache_append
    kv = _packed(T=3, H=2)

    def call(c=None, k=kv, v=kv, cu=None):
        return f(R(c or _cache()), R(k), R(v), cu, None)

    assert f(None, R(kv), R(kv), None, None) == NULL and f(R(_cache()), None, R(kv), None, None) == NULL and f(R(_cache()), R(kv), None, None, None) == NULL
    assert call(k=_packed(T=3, H=2, dtype=F32)) == DTYPE and call(v=_packed(T=3, H=2, dtype=F32)) == DTYPE
    assert call(k=_packed(T=3, H=4)) == SHAPE and call(v=_packed(T=4, H=2)) == SHAPE and call(k=_packed(T=3, H=2, D=64)) == SHAPE
    assert call(k=_packed(T=4, H=2), v=_packed(T=4, H=2)) == SHAPE
    assert call(k=_packed(T=3, H=2, sl=100)) == STRIDE
    assert call(c=_cache(n_seqs=0), k=_packed(T=0, H=2, data=None), v=_packed(T=0, H=2, data=None)) == 0
    assert call(c=_cache(max_pages=0, table=None, stride=0)) == 0


def test_validate_refusals():
    f = binding.load_library().sparsed_cache_validate
    assert f(None, None) == NULL and f(R(_cache()), None) == WORKSPACE and f(R(_cache(stride=3)), R(_ex())) == STRIDE
    assert f(R(_cache(n_seqs=0)), R(_ex())) == 0


def test_workspace_size_and_its_arguments():
    f = binding.load_library().sparsed_paged_workspace_bytes
    assert f(None, R(_cache())) == 0 and f(R(_packed()), None) == 0 and f(R(_packed(H=0)), R(_cache())) == 0
    small, large = f(R(_packed(T=1)), R(_cache())), f(R(_packed(T=64)), R(_cache()))
    assert 0 < small <= large and small % 256 == 0 and large % 256 == 0


def test_packed_cache_struct_matches_its_mirror():
    k, v = (0x7fff00000100, 0, 5, 6, 7, 8, 1 << 40, 9, 10), (0x7fff00000200, 1, 15, 16, 17, 18, -3, 19, 20)
    rest = (0x7fff00000300, 0x7fff00000400, 21, 22, 1 << 35)
    raw = binding._pack_tensor(*k) + binding._pack_tensor(*v) + binding._pack_table(*rest)
    assert len(raw) == ctypes.sizeof(binding._PagedCache)
    c = binding._PagedCache.from_buffer_copy(raw)
    assert [getattr(c.k, f[0]) for f in c.k._fields_] == list(k) and [getattr(c.v, f[0]) for f in c.v._fields_] == list(v)
    assert (c.page_table, c.seq_lens, c.n_seqs, c.max_pages, c.table_stride) == rest


def test_python_arguments():
    """Tensors that are no tensors of the right kind are refused before anything else happens."""
    import paper_2509_24014_amd as sd
    x, cu = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.tensor([0, 4], dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sd.attn_prompt(x, x, x, cu)
    with pytest.raises(ValueError, match=r"\[T, H, D\]"):
        sd.attn_prompt(x[None], x, x, cu)
    with pytest.raises(ValueError, match="bf16 or fp32"):
        sd.attn_prompt(x.half(), x, x, cu)
    with pytest.raises(ValueError, match="contiguous"):
        sd.attn_prompt(x.transpose(1, 2), x, x, cu)
    pages, table, lens = torch.zeros(3, 16, 2, 64), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sd.PagedCache(pages, pages, table, lens)
    with pytest.raises(ValueError, match="n_pages"):
        sd.PagedCache(pages[0], pages, table, lens)
