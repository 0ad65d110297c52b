"""What a wait of wnw_pages_attend that runs out leaves behind.  The debug hook has kernels wait for what never happens, for half a
millisecond; a kernel starts nothing behind such a wait and goes on only when what it has under way is at rest, so no GPU is put at risk."""
import pytest
import torch

import paper_2608_22704_b200 as wnw
from pages_ref import E4M3, INT8
from test_gpu_pages import DEV, attend, filled, randn

PROMPT = ["K_FREE", "V_FREE", "K_FULL", "V_FULL", "Q_FULL", "SCORES", "WEIGHTS", "VALUES", "BEGUN", "ALL"]


def test_waits_that_there_are_not():
    for waits in (-1, 1 << 20):
        with pytest.raises(wnw.WnwError) as e:
            wnw.wnw_debug_pages_lose(waits)
        assert e.value.status == wnw.WNW_ERR_INVALID_ARG
    wnw.wnw_debug_pages_lose(0)


def lost(b, lengths, rows, q, waits, **how):
    """A call whose waits of these kinds run out: (out, lse, the status word)."""
    b.status.zero_()
    wnw.wnw_debug_pages_lose(waits)
    try:
        out, lse = attend(b.pages, b.table_dev, lengths, rows, q, **how)
        torch.cuda.synchronize()
    finally:
        wnw.wnw_debug_pages_lose(0)
    status = b.status.item()
    b.status.zero_()
    return out, lse, status


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,d", [(E4M3, 64), (INT8, 128)])
@pytest.mark.parametrize("waits", PROMPT)
def test_rows_of_a_prompt_whose_wait_runs_out_are_not_a_numbers(fmt, d, waits):
    """Many tiles and segments to a CTA, items of one and of two row tiles, items that CTAs share.  A row is complete or not a number; and
    where a CTA loses the first wait of the kind that it makes for its rows, none is complete.  (Room for the first tiles is there from
    the start, and BEGUN is the wait of a row tile without rows: those find some rows complete.)"""
    lengths, rows = [3000, 1400, 40, 2000], [70, 20, 20, 130]
    n = sum(rows)
    b = filled(fmt, 8, 64, d, lengths, seed=5)
    q = randn(n + 2, 32, d, seed=9, scale=2.0).to(DEV)
    for causal in (True, False):
        want, want_lse = attend(b.pages, b.table_dev, lengths, rows, q, causal=causal)
        assert want[:n].isfinite().all()
        out, lse, status = lost(b, lengths, rows, q, getattr(wnw, "WNW_DEBUG_WAIT_" + waits), causal=causal)
        assert status == wnw.WNW_PAGES_TIMEOUT
        gone = out[:n].isnan().all(-1)
        assert torch.equal(gone, lse[:n].isnan())
        assert gone.any() if waits in ("K_FREE", "V_FREE", "BEGUN") else gone.all()
        assert torch.equal(out[:n][~gone], want[:n][~gone]) and torch.equal(lse[:n][~gone], want_lse[:n][~gone])
        assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
        again, again_lse = attend(b.pages, b.table_dev, lengths, rows, q, causal=causal)         # the next call is as if nothing had been
        assert torch.equal(again, want) and torch.equal(again_lse, want_lse) and b.status.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,hq,heads,d", [(E4M3, 32, 8, 128), (INT8, 8, 4, 64)])
@pytest.mark.parametrize("rows,wide", [(1, False), (1, True), (4, False), (4, True)])
def test_rows_of_a_copy_that_does_not_arrive_are_not_a_numbers(fmt, hq, heads, d, rows, wide):
    """In clusters and on the line, where a CTA goes on to other heads: every row that sees a token lacks one.  One that sees none is complete
    unless it shares a CTA with those."""
    lengths = [900, 0, 5000 if wide else 300, 17]
    b = filled(fmt, heads, 64, d, lengths, seed=5)
    q = randn(4 * rows + 2, hq, d, seed=9, scale=2.0).to(DEV)
    if wide:
        table = torch.full((4, 1 << 16), 10 ** 9, dtype=torch.int32, device=DEV)                 # never looked at
        table[:, :b.table_dev.shape[1]] = b.table_dev
        b.table_dev = table
    n = 4 * rows
    sees = torch.tensor([s != 1 for s in range(4) for _ in range(rows)], device=DEV)
    want, want_lse = attend(b.pages, b.table_dev, lengths, [rows] * 4, q, max_rows=rows)
    assert want[:n].isfinite().all()
    out, lse, status = lost(b, lengths, [rows] * 4, q, wnw.WNW_DEBUG_WAIT_GRANULE, max_rows=rows)
    assert status == wnw.WNW_PAGES_TIMEOUT
    gone = out[:n].isnan().all(-1)
    assert torch.equal(gone, lse[:n].isnan()) and gone[sees].all()
    assert (out[:n][~gone] == 0).all() and lse[:n][~gone].isneginf().all()
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
    again, again_lse = attend(b.pages, b.table_dev, lengths, [rows] * 4, q, max_rows=rows)
    assert torch.equal(again, want) and torch.equal(again_lse, want_lse) and b.status.item() == 0
