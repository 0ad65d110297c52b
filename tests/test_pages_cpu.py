"""Rotary plans, and what the calls around the paged store refuse before they touch the device (no GPU needed)."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_22704_b200 as wnw
from pages_ref import E4M3, HIGHEST, INT8, LARGEST, LOWEST, exponent_for, nearest_code


def test_rotary_plan_of_consecutive_runs():
    r = wnw.wnw_rotary_init(64, 1e6, [16, 24, 24])
    assert (r.n_pairs, r.n_axes, r.neighbours) == (64, 3, 0)
    assert list(r.axis)[:64] == [0] * 16 + [1] * 24 + [2] * 24
    for i in (0, 1, 31, 63):
        assert r.frequency[i] == pytest.approx(1e6 ** (-i / 64), rel=1e-14)


def test_rotary_plan_dealt_in_turn():
    r = wnw.wnw_rotary_init(10, 1e4, [6, 3, 1], dealt=True, neighbours=True)
    # turns 0 1 2 0 1 2 0 1 2 0: the third axis has one pair, the second three
    assert list(r.axis)[:10] == [0, 1, 2, 0, 1, 0, 0, 1, 0, 0]
    assert r.neighbours == 1


def test_rotary_plan_with_an_axis_of_no_pairs():
    assert list(wnw.wnw_rotary_init(4, 1e4, [0, 3, 0, 1]).axis)[:4] == [1, 1, 1, 3]


@pytest.mark.parametrize("args", [(0, 1e4, [0]), (129, 1e4, [129]), (8, 0.0, [8]), (8, math.inf, [8]), (8, 1e4, [4, 3]), (8, 1e4, [9, -1]),
                                  (8, 1e4, [2, 2, 2, 1, 1])])
def test_rotary_plan_refusals(args):
    with pytest.raises(wnw.WnwError) as e:
        wnw.wnw_rotary_init(*args)
    assert e.value.status == wnw.WNW_ERR_INVALID_ARG


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_scale_brings_the_largest_magnitude_into_the_top_binade(fmt):
    rs = np.random.RandomState(1)
    for _ in range(500):
        x = rs.randn(7) * 2.0 ** rs.randint(-100, 100)
        e = exponent_for(x, fmt)
        top = np.abs(x).max() / 2.0 ** e
        assert LARGEST[fmt] / 2 < top <= LARGEST[fmt] or e == LOWEST
        assert np.abs(nearest_code(np.ldexp(x, -e), fmt)).max() <= LARGEST[fmt]
    assert exponent_for(np.zeros(3), fmt) == LOWEST and exponent_for([3e38], fmt) <= HIGHEST[fmt]


# ---- refusals: the pointers are never followed ----
def test_calls_are_packed_as_the_structures_are():
    from paper_2608_22704_b200 import binding
    for call, structure in ((binding._rotate_call, wnw.wnw_rotate_t), (binding._rows_call, wnw.wnw_pages_rows_t),
                            (binding._attend_call, wnw.wnw_pages_attend_t)):
        assert call.size == C.sizeof(structure)
    n = iter(range(1, 100))
    a = wnw.wnw_pages_attend_t.from_buffer_copy(binding._attend_call.pack(*[next(n) for _ in range(26)]))
    assert (a.pages, a.batch.page_table_dev, a.batch.max_rows, a.q.dev, a.q.n_heads, a.out.row_stride) == (1, 2, 8, 9, 12, 15)
    assert (a.lse_dev, a.workspace_bytes, a.dtype, a.causal, a.softmax_scale, a.cuda_stream) == (19, 21, 22, 23, 24.0, 26)


def _pages(**kw):
    args = dict(codes_dev=1 << 20, scales_dev=1 << 20, page_stride=0, scale_stride=0, n_pages=8, page_tokens=64, n_kv_heads=4, head_dim=128,
                format=0, device=0, status_dev=None)
    args.update(kw)
    return wnw.wnw_pages_t(*args.values())


def _batch(**kw):
    args = dict(page_table_dev=1 << 20, lengths_dev=1 << 20, row_starts_dev=1 << 20, table_stride=4, n_seqs=2, n_rows=2, max_rows=1)
    args.update(kw)
    return wnw.wnw_batch_t(*args.values())


def _rows(heads=4, dim=128, **kw):
    args = dict(dev=1 << 20, row_stride=heads * dim, head_stride=dim, n_heads=heads, reserved=0)
    args.update(kw)
    return wnw.wnw_rows_t(*args.values())


def _all(pages=None, batch=None, k=None, v=None, q=None, out=None, dtype=0, causal=1, scale=0.0, workspace=1 << 20, size=1 << 30):
    """The statuses of write, read and attend."""
    lib, pages, batch = wnw.lib(), pages or _pages(), batch or _batch()
    rows = C.byref(wnw.wnw_pages_rows_t(C.addressof(pages), batch, k or _rows(), v or _rows(), None, None, 0, dtype, 0, None))
    call = wnw.wnw_pages_attend_t(C.addressof(pages), batch, q or _rows(16), out or _rows(16), None, workspace, size, dtype, causal, scale, 0, None)
    return lib.wnw_pages_write(rows), lib.wnw_pages_read(rows), lib.wnw_pages_attend(C.byref(call))


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), "UNSUPPORTED"), (dict(page_tokens=8), "UNSUPPORTED"), (dict(page_tokens=72), "UNSUPPORTED"),
    (dict(page_tokens=272), "UNSUPPORTED"), (dict(n_kv_heads=0), "INVALID_ARG"), (dict(n_kv_heads=1025), "CAPACITY"),
    (dict(format=2), "INVALID_ARG"), (dict(n_pages=-1), "INVALID_ARG"), (dict(codes_dev=None), "INVALID_ARG"),
    (dict(codes_dev=(1 << 20) + 8), "INVALID_ARG"), (dict(scales_dev=(1 << 20) + 2), "INVALID_ARG"), (dict(page_stride=64 * 128), "INVALID_ARG"),
    (dict(page_stride=(1 << 20) + 8), "INVALID_ARG"), (dict(scale_stride=7), "INVALID_ARG"), (dict(status_dev=(1 << 20) + 1), "INVALID_ARG"),
])
def test_stores_that_are_refused(kw, status):
    assert _all(pages=_pages(**kw)) == (getattr(wnw, "WNW_ERR_" + status),) * 3


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=-1), "INVALID_ARG"), (dict(n_seqs=1025), "CAPACITY"), (dict(n_rows=-1), "INVALID_ARG"), (dict(max_rows=-1), "INVALID_ARG"),
    (dict(lengths_dev=None), "INVALID_ARG"), (dict(row_starts_dev=None), "INVALID_ARG"), (dict(page_table_dev=None), "INVALID_ARG"),
    (dict(table_stride=-1), "INVALID_ARG"), (dict(table_stride=1 << 25), "CAPACITY"), (dict(lengths_dev=(1 << 20) + 2), "INVALID_ARG"),
])
def test_batches_that_are_refused(kw, status):
    assert _all(batch=_batch(**kw)) == (getattr(wnw, "WNW_ERR_" + status),) * 3


def test_rows_that_are_refused():
    bad, unsup = wnw.WNW_ERR_INVALID_ARG, wnw.WNW_ERR_UNSUPPORTED
    for kw in (dict(dev=None), dict(dev=(1 << 20) + 2), dict(row_stride=516), dict(head_stride=132)):
        rows, rows16 = _rows(**kw), _rows(16, **kw)
        assert _all(k=rows)[:2] == (bad, bad) and _all(v=rows)[:2] == (bad, bad)
        assert _all(q=rows16)[2] == bad and _all(out=rows16)[2] == bad
    assert _all(k=_rows(3))[:2] == (bad, bad)
    assert _all(q=_rows(6), out=_rows(6))[2] == bad and _all(q=_rows(16), out=_rows(8))[2] == bad
    assert _all(q=_rows(68), out=_rows(68))[2] == unsup                # a group of 17
    assert _all(dtype=2) == (unsup,) * 3 and _all(dtype=-1) == (unsup,) * 3
    assert _all(causal=2)[2] == bad and _all(scale=-1.0)[2] == bad and _all(scale=math.nan)[2] == bad and _all(scale=math.inf)[2] == bad


def test_nothing_to_do_is_no_error():
    ok = (wnw.WNW_OK,) * 3
    assert _all(batch=_batch(n_seqs=0)) == ok
    assert _all(batch=_batch(n_rows=0), k=_rows(dev=None), v=_rows(dev=None), q=_rows(16, dev=None), out=_rows(16, dev=None)) == ok


def test_null_arguments():
    lib, bad = wnw.lib(), wnw.WNW_ERR_INVALID_ARG
    assert lib.wnw_rotate(None) == lib.wnw_pages_write(None) == lib.wnw_pages_read(None) == lib.wnw_pages_attend(None) == bad
    rows = wnw.wnw_pages_rows_t(None, _batch(), _rows(), _rows(), None, None, 0, 0, 0, None)
    assert lib.wnw_pages_write(C.byref(rows)) == lib.wnw_pages_read(C.byref(rows)) == bad
    call = wnw.wnw_pages_attend_t(None, _batch(), _rows(16), _rows(16), None, 1 << 20, 1 << 30, 0, 1, 0.0, 0, None)
    assert lib.wnw_pages_attend(C.byref(call)) == bad
    n, p = C.c_int64(5), C.byref(_pages())
    assert lib.wnw_pages_attend_workspace(None, 16, C.byref(n)) == bad and lib.wnw_pages_attend_workspace(p, 16, None) == bad
    assert lib.wnw_pages_attend_workspace(p, 7, C.byref(n)) == bad and n.value == 5


def test_rotary_of_a_write():
    lib, pages = wnw.lib(), _pages()

    def write(r, at=1 << 20, call=lib.wnw_pages_write):
        return call(C.byref(wnw.wnw_pages_rows_t(C.addressof(pages), _batch(), _rows(), _rows(), C.addressof(r), at, 2, 0, 0, None)))

    assert write(wnw.wnw_rotary_init(65, 1e4)) == wnw.WNW_ERR_INVALID_ARG            # more elements than a head has
    assert write(wnw.wnw_rotary_init(20, 1e4)) == wnw.WNW_ERR_UNSUPPORTED            # not in eights
    assert write(wnw.wnw_rotary_init(64, 1e4), None) == wnw.WNW_ERR_INVALID_ARG
    assert write(wnw.wnw_rotary_init(64, 1e4), call=lib.wnw_pages_read) == wnw.WNW_ERR_INVALID_ARG
    r = wnw.wnw_rotary_init(64, 1e4)
    r.axis[3] = 1
    assert write(r) == wnw.WNW_ERR_INVALID_ARG                                       # an axis that is not there
    r = wnw.wnw_rotary_init(64, 1e4)
    r.frequency[9] = math.nan
    assert write(r) == wnw.WNW_ERR_INVALID_ARG


def test_rotate_refusals():
    lib = wnw.lib()

    def rotate(r=None, q=None, q_out=None, k=None, k_out=None, n=3, d=128, dtype=0, inverse=0, at=1 << 20):
        none = _rows(dev=None)
        r = r or wnw.wnw_rotary_init(d // 2 if 0 < d <= 256 else 1, 1e4)
        return lib.wnw_rotate(C.byref(wnw.wnw_rotate_t(C.addressof(r), at, n, q or _rows(), q_out or _rows(), k or none, k_out or none, n, d, dtype, inverse,
                                                       0, 0, None)))

    bad, unsup = wnw.WNW_ERR_INVALID_ARG, wnw.WNW_ERR_UNSUPPORTED
    assert rotate(n=-1) == bad and rotate(inverse=2) == bad and rotate(at=None) == bad
    assert rotate(k=_rows()) == bad and rotate(k_out=_rows()) == bad
    assert rotate(r=wnw.wnw_rotary_init(65, 1e4)) == bad
    assert rotate(q=_rows(3)) == bad and rotate(q=_rows(dev=None)) == bad and rotate(q=_rows(dev=(1 << 20) + 1)) == bad
    assert rotate(dtype=3) == unsup and rotate(d=258) == unsup and rotate(d=0) == unsup
    assert rotate(n=0) == wnw.WNW_OK and rotate(n=0, at=None) == wnw.WNW_OK
