"""Calls around the paged store at the edges of what they allow (needs a B200)."""
import pytest
import torch

import paper_2608_22704_b200 as wnw
from test_gpu_pages import DEV, attend, ints, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("rows", [1, 20])
def test_a_store_of_no_pages(fmt, rows):
    """Every page id lies outside it: nothing is written, zeros are read, nothing is attended to."""
    heads, hq, T, d = 2, 8, 16, 64
    status = ints([0])
    pages = wnw.wnw_pages(torch.empty(0, heads, 2, T, d, dtype=fmt, device=DEV), torch.empty(0, heads, 2, device=DEV), status)
    table = ints([[0, 1], [0, 0]])
    k, v = (randn(2 * rows, heads, d, seed=s).to(DEV) for s in (1, 2))
    wnw.wnw_pages_write(pages, table, ints([0, 0]), ints([0, rows, 2 * rows]), k, v)
    assert status.item() == wnw.WNW_PAGES_BAD_PAGE
    wnw.wnw_pages_read(pages, table, ints([0, 0]), ints([0, rows, 2 * rows]), k, v)
    assert (k == 0).all() and (v == 0).all()
    for wide in (False, True):
        if wide:
            table = torch.zeros(2, 1 << 18, dtype=torch.int32, device=DEV)
        out, lse = attend(pages, table, [30, 0], [rows, rows], randn(2 * rows, hq, d, seed=3).to(DEV), max_rows=rows)
        assert (out == 0).all() and lse.isneginf().all()
        assert status.item() == wnw.WNW_PAGES_BAD_PAGE
