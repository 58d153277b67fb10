"""What the cache calls refuse: their Python face before anything reaches the library, and the C entry points by the strides of what they
write. Nothing here needs a GPU."""
import ctypes
import types

import pytest
import torch

import paper_2509_24014_amd as sd
from paper_2509_24014_amd import binding

PAGES = torch.zeros(6, 16, 2, 64)
LENS = torch.zeros(3, dtype=torch.int32)


def _cache(table, lens=LENS):
    return sd.PagedCache(PAGES, PAGES, table, lens)


def test_rows_of_a_page_table_that_lie_closer_than_they_are_long():
    """A row shared by all sequences (stride 0), or rows that overlap: the kernels step from row to row by the stride."""
    shared = torch.arange(4, dtype=torch.int32)[None].expand(3, -1)
    overlapping = torch.arange(9, dtype=torch.int32).as_strided((3, 4), (2, 1))
    one_page = torch.zeros(1, 1, dtype=torch.int32).expand(3, -1)
    for table in (shared, overlapping, one_page):
        with pytest.raises(ValueError, match="rows of page_table"):
            _cache(table)


def test_page_tables_with_rows_apart_pass_on():
    """The next refusal is that of pages in host memory."""
    wide = torch.zeros(3, 10, dtype=torch.int32)
    for table, lens in ((wide, LENS), (wide[:, :4], LENS), (wide[:, :1], LENS), (wide[:, :0], LENS), (wide[:1].expand(1, -1), LENS[:1]),
                        (torch.zeros(3, 1, dtype=torch.int32), LENS), (torch.zeros(8, dtype=torch.int32).as_strided((1, 4), (0, 1)), LENS[:1])):
        with pytest.raises(ValueError, match="GPU"):
            _cache(table, lens)


# ---- the C entry points: rows that are written must not share memory


def _packed(T, H, D, sl, sh):
    return binding._Tensor(0x1000, binding.SPARSED_BF16, 1, H, T, D, 0, sh, sl)


@pytest.mark.parametrize("sl,sh,apart", [(4 * 64, 64, True), (64, 100 * 64, True), (64, 99 * 64, False), (64, 64, False), (3 * 64, 64, False),
                                         (512, 64, True), (4 * 64, 0, False), (4 * 64, 1 << 40, True), (128, 64, False)])
def test_rows_of_an_output(sl, sh, apart):
    lib, R = binding.load_library(), ctypes.byref
    q, kv, out = _packed(100, 4, 64, 256, 64), _packed(100, 2, 64, 128, 64), _packed(100, 4, 64, sl, sh)
    # no sequences: nothing runs where nothing is refused
    assert lib.sparsed_attn_prompt(R(q), R(kv), R(kv), R(out), None, None, 0, 1, None) == (0 if apart else 4)
    pages = binding._Tensor(0x2000, binding.SPARSED_BF16, 5, 2, 16, 64, 16 * 128, 64, 128)
    cache = binding._PagedCache(pages, pages, None, None, 0, 0, 0)
    assert lib.sparsed_attn_paged(R(q), R(cache), 0x5000, 1, R(out), None) == (0 if apart else 4)


def test_one_token_or_one_head_of_an_output_may_have_any_stride():
    lib, R = binding.load_library(), ctypes.byref
    for T, H, sl, sh in ((1, 4, 0, 64), (100, 1, 64, 0), (1, 1, 0, 0), (0, 4, 0, 0)):
        q, kv = _packed(T, H, 64, 64 * H, 64), _packed(T, 1, 64, 64, 64)
        assert lib.sparsed_attn_prompt(R(q), R(kv), R(kv), R(_packed(T, H, 64, sl, sh)), None, None, 0, 1, None) == 0


@pytest.mark.parametrize("n,H,sb,sh,sl,apart", [(5, 2, 2048, 64, 128, True), (5, 2, 2048, 1024, 64, True), (5, 2, 1024, 5 * 1024, 64, True),
                                                (5, 2, 2 * 2048, 64, 128, True), (5, 2, 2048, 0, 128, False), (5, 2, 0, 64, 128, False),
                                                (5, 2, 1024, 64, 128, False), (1, 2, 0, 64, 128, True), (5, 1, 1024, 0, 64, True),
                                                (5, 2, 2048, 64, 64, False), (5, 2, 1984, 64, 128, False)])
def test_places_of_a_cache(n, H, sb, sh, sl, apart):
    """Append writes them; attention, which reads them, takes any."""
    lib, R = binding.load_library(), ctypes.byref
    good = binding._Tensor(0x2000, binding.SPARSED_BF16, n, H, 16, 64, 16 * 64 * H, 64, 64 * H)
    pages = binding._Tensor(0x2000, binding.SPARSED_BF16, n, H, 16, 64, sb, sh, sl)
    kv, q = _packed(0, H, 64, 64 * H, 64), _packed(0, 4, 64, 256, 64)
    for k, v in ((pages, good), (good, pages)):
        cache = binding._PagedCache(k, v, None, None, 0, 0, 0)
        assert lib.sparsed_cache_append(R(cache), R(kv), R(kv), None, None) == (0 if apart else 4)
        assert lib.sparsed_attn_paged(R(q), R(cache), None, 1, R(q), None) == 0


def test_log_sum_exp_in_another_order():
    """[Hq, T] is what the kernels fill; a [T, Hq] tensor of as many elements is not it."""
    q, host = torch.zeros(6, 4, 64), torch.device("cpu")
    assert binding._lse_ptr(torch.zeros(4, 6), q, host) != 0
    for bad in (torch.zeros(6, 4), torch.zeros(24), torch.zeros(1, 4, 6), torch.zeros(4, 6, dtype=torch.float64), torch.zeros(4, 12)[:, :6],
                torch.zeros(6, 4).t(), torch.zeros(4, 5)):
        with pytest.raises(ValueError, match=r"\[Hq, T\]"):
            binding._lse_ptr(bad, q, host)


def test_more_sequences_than_an_attention_call_takes():
    """Every work-group looks through all of them: a million would take minutes. Append and validation do not care."""
    lib, R, none = binding.load_library(), ctypes.byref, _packed(0, 2, 64, 128, 64)
    pages = binding._Tensor(0x2000, binding.SPARSED_BF16, 5, 2, 16, 64, 16 * 128, 64, 128)
    for n, status in ((1 << 16, 0), ((1 << 16) + 1, 6), (1 << 20, 6), (1 << 30, 6)):
        cache = binding._PagedCache(pages, pages, 0x3000, 0x4000, n, 1, 1)
        assert lib.sparsed_attn_prompt(R(none), R(none), R(none), R(none), 0x5000, None, n, 1, None) == status
        assert lib.sparsed_attn_paged(R(none), R(cache), 0x5000, 1, R(none), None) == status
        assert (lib.sparsed_paged_workspace_bytes(R(none), R(cache)) > 0) == (status == 0)
        assert lib.sparsed_cache_append(R(cache), R(none), R(none), 0x5000, None) == 0


def test_a_stream_of_another_device():
    """Before anything is launched; the device of the tensors need not be the current one."""
    calls = []
    with pytest.raises(ValueError, match="stream is on cuda:1"):
        binding._launch(torch.device("cuda", 0), lambda *a: calls.append(a), stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    assert not calls
