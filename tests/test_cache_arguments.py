"""What the Python face of the cache calls refuses before anything reaches the library: nothing here needs a GPU."""
import pytest
import torch

import paper_2509_24014_amd as sd

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
