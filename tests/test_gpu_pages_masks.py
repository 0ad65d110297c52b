"""What a row of wnw_pages_attend does not see does not reach it: the forms for few query rows, against float64 (needs a B200)."""
import pytest
import torch

from pages_ref import E4M3
from test_gpu_pages import DEV, Both, attend, check_attention, randn, values_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,heads,d,T", [(8, 2, 128, 32), (10, 1, 64, 16), (32, 2, 128, 64), (4, 4, 64, 48)])
@pytest.mark.parametrize("rows", [2, 3, 5])
@pytest.mark.parametrize("wide", [False, True])
def test_not_a_numbers_of_later_rows_stay_with_them(hq, heads, d, T, rows, wide):
    """V's (and K's) not-a-numbers at the tokens of a sequence's last rows: in the last granule of every row, at its border, in one of its
    own.  Items of one query token (a group of more than eight, or max_rows = 1) stand before the others of their sequence; a table as wide as
    a pool's sends the call from the clusters to the line."""
    lengths = [150, 145, 16, rows]
    width = max((n + T - 1) // T for n in lengths)
    for at_k, at_v in ((None, 1), (None, 2), (1, rows)):                       # tokens from a sequence's end
        b = Both(4 * width, heads, T, d, E4M3, 4, width)
        k, v = randn(sum(lengths), heads, d, seed=1).to(DEV), randn(sum(lengths), heads, d, seed=2).to(DEV)
        end = 0
        for n in lengths:
            end += n
            v[end - at_v, 0, 7] = float("nan")
            v[end - at_v, heads - 1, d - 1] = float("nan")
            if at_k is not None:
                k[end - at_k, heads - 1, 5] = float("nan")
        b.write(k, v, lengths)
        b.check()
        q = randn(4 * rows + 1, hq, d, seed=3).to(DEV)
        table = b.table_dev
        if wide:
            table = torch.full((4, (1 << 22) // T), 10 ** 9, dtype=torch.int32, device=DEV)       # never looked at
            table[:, :width] = b.table_dev
        for max_rows in (0, 1, rows):
            for causal in (True, False):
                out, lse = attend(b.pages, table, lengths, [rows] * 4, q, causal=causal, max_rows=max_rows)
                check_attention(out, lse, q, values_of(b, lengths), lengths, [rows] * 4, causal, T=T)
    assert b.status.item() == 0
