"""What the calls of the paged cache refuse, on the host before anything is launched (CPU only)."""
import ctypes as C
import os

import pytest
import torch

from paper_2602_21780_amd import xsv


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(xsv.LIB_PATH):
        from paper_2602_21780_amd.build import build
        build()
    return xsv.lib()


PTR = 1 << 20    # an aligned address that nothing looks at
T = xsv.xsv_tensor(PTR, 4 * 64, 64)
NONE = xsv.xsv_tensor(None, 0, 0)
BAD_TENSORS = [xsv.xsv_tensor(None, 256, 64), xsv.xsv_tensor(PTR + 8, 256, 64), xsv.xsv_tensor(PTR, 256, 60), xsv.xsv_tensor(PTR, 256, 68),
               xsv.xsv_tensor(PTR, -256, 64), xsv.xsv_tensor(PTR, 4, 64), xsv.xsv_tensor(PTR, 256, (1 << 24) + 8)]


def _pages(**kw):
    good = dict(pages=9, kv_heads=2, k=PTR, v=PTR, k_scale=PTR, v_scale=PTR, k_bounds=PTR, sequences=1, table_width=4, table=PTR, lengths=PTR)
    return xsv.xsv_pages(**{**good, **kw})


def _query(**kw):
    good = dict(heads=4, rows=8, longest_q=8, longest_k=256, q_begin=PTR, causal=0, softmax_scale=0.0, chosen=None, count=3, first=1, last=1)
    return xsv.xsv_pages_query(**{**good, **kw})


def _calls(lib, p, c, begin=PTR, rows=8, longest=8, t=T):
    nbytes = C.c_int64()
    p, c = C.byref(p), C.byref(c)
    return [lib.xsv_pages_write(None, p, begin, rows, longest, t, t), lib.xsv_pages_read(None, p, begin, rows, longest, t, t),
            lib.xsv_pages_attend_workspace(p, c, C.byref(nbytes)), lib.xsv_pages_attend(None, p, c, t, t, PTR, PTR, 1 << 40),
            lib.xsv_pages_select(None, p, c, t, PTR)]


@pytest.mark.parametrize("bad", [dict(pages=-1), dict(kv_heads=0), dict(kv_heads=-2), dict(k=None), dict(v=None), dict(k_scale=None), dict(v_scale=None),
                                 dict(k=PTR + 8), dict(v=PTR + 4), dict(k_scale=PTR + 2), dict(v_scale=PTR + 1), dict(k_bounds=PTR + 8), dict(sequences=-1),
                                 dict(table_width=-1), dict(table=None), dict(lengths=None), dict(table=PTR + 2), dict(lengths=PTR + 3)])
def test_pools_that_are_refused(lib, bad):
    assert _calls(lib, _pages(**bad), _query()) == [xsv.XSV_ERR_ARG] * 5


@pytest.mark.parametrize("bad", [dict(heads=0), dict(heads=3), dict(heads=-2), dict(rows=-1), dict(longest_q=9), dict(longest_q=-1), dict(longest_k=-1),
                                 dict(q_begin=None), dict(q_begin=PTR + 2), dict(causal=-1), dict(softmax_scale=-1.0), dict(softmax_scale=1e-30),
                                 dict(softmax_scale=1e30), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(count=-1),
                                 dict(first=-1), dict(last=-1), dict(chosen=PTR + 2)])
def test_questions_that_are_refused(lib, bad):
    assert _calls(lib, _pages(), _query(**bad))[2:] == [xsv.XSV_ERR_ARG] * 3


def test_rows_tensors_and_workspaces_that_are_refused(lib):
    p, c = C.byref(_pages()), _query()
    for kw in (dict(begin=None), dict(begin=PTR + 1), dict(rows=-1), dict(longest=9), dict(longest=-1)):
        assert _calls(lib, _pages(), c, **kw)[:2] == [xsv.XSV_ERR_ARG] * 2
    for bad in BAD_TENSORS:
        for x, y in ((bad, T), (T, bad)):
            assert lib.xsv_pages_write(None, p, PTR, 8, 8, x, y) == xsv.XSV_ERR_ARG
            assert lib.xsv_pages_read(None, p, PTR, 8, 8, x, y) == xsv.XSV_ERR_ARG
            assert lib.xsv_pages_attend(None, p, C.byref(c), x, y, PTR, PTR, 1 << 40) == xsv.XSV_ERR_ARG
        assert lib.xsv_pages_select(None, p, C.byref(c), bad, PTR) == xsv.XSV_ERR_ARG
    for lse in (None, PTR + 2):
        assert lib.xsv_pages_attend(None, p, C.byref(c), T, T, lse, PTR, 1 << 40) == xsv.XSV_ERR_ARG
    for chosen in (None, PTR + 2):
        assert lib.xsv_pages_select(None, p, C.byref(c), T, chosen) == xsv.XSV_ERR_ARG
    long = _query(rows=1, longest_q=1, longest_k=1 << 20)
    pages = _pages(table_width=1 << 14)
    nbytes = C.c_int64()
    assert lib.xsv_pages_attend_workspace(C.byref(pages), C.byref(long), None) == xsv.XSV_ERR_ARG
    assert lib.xsv_pages_attend_workspace(C.byref(pages), C.byref(long), C.byref(nbytes)) == xsv.XSV_OK and nbytes.value > 0
    for work, size in ((None, nbytes.value), (PTR, nbytes.value - 1), (PTR + 8, nbytes.value)):
        assert lib.xsv_pages_attend(None, C.byref(pages), C.byref(long), T, T, PTR, work, size) == xsv.XSV_ERR_ARG


def test_choices_that_are_refused(lib):
    p = C.byref(_pages())
    for bad in (dict(count=0, first=0, last=0), dict(count=3, first=2, last=2), dict(count=1, first=(1 << 31) - 1, last=(1 << 31) - 1)):
        assert lib.xsv_pages_select(None, p, C.byref(_query(**bad)), T, PTR) == xsv.XSV_ERR_ARG
    assert lib.xsv_pages_select(None, C.byref(_pages(k_bounds=None)), C.byref(_query()), T, PTR) == xsv.XSV_ERR_ARG
    many = _pages(table_width=40000)
    assert lib.xsv_pages_select(None, C.byref(many), C.byref(_query(longest_k=32769 * 64)), T, PTR) == xsv.XSV_ERR_UNSUPPORTED


def test_sizes_that_are_not_supported(lib):
    U = xsv.XSV_ERR_UNSUPPORTED
    assert _calls(lib, _pages(kv_heads=(1 << 16) + 1), _query(heads=(1 << 16) + 1)) == [U] * 5
    assert _calls(lib, _pages(table_width=(1 << 24) + 1), _query()) == [U] * 5
    assert _calls(lib, _pages(), _query(heads=1 << 17))[2:] == [U] * 3
    assert _calls(lib, _pages(), _query(count=(1 << 24) + 1))[2:] == [U] * 3
    big = (1 << 31) - 1
    assert _calls(lib, _pages(sequences=big), _query(rows=big, longest_q=big), rows=big, longest=big) == [U] * 5
    assert _calls(lib, _pages(kv_heads=1 << 16, sequences=big), _query(heads=1 << 16, rows=big, longest_q=big), rows=big, longest=big) == [U] * 5


def test_nothing_to_do_needs_no_tensors(lib):
    for p, c, rows in ((_pages(sequences=0, table=None, lengths=None), _query(rows=0, longest_q=0, q_begin=None), 0),
                       (_pages(), _query(rows=0, longest_q=0), 0),
                       (_pages(pages=0, k=None, v=None, k_scale=None, v_scale=None, k_bounds=None, sequences=0, table=None, lengths=None, table_width=0),
                        _query(rows=0, longest_q=0, q_begin=None), 0)):
        assert _calls(lib, p, c, rows=rows, longest=0, t=NONE) == [xsv.XSV_OK] * 5


def test_bindings_refuse_tensors_that_are_not_a_pool():
    host = lambda *shape, dtype: torch.zeros(shape, dtype=dtype)
    with pytest.raises(ValueError):
        xsv.Pages(host(2, 2, 64, 64, dtype=torch.float32), None, None, None)
    with pytest.raises(ValueError):
        xsv.Pages.empty(2, 2, "cpu")
    with pytest.raises(ValueError):
        xsv.Pages(None, None, None, None)


def test_launches_are_sized_by_the_rows_and_the_sequences(lib):
    """Not by the rows of all that one sequence may have, for each of them."""
    nbytes = C.c_int64()
    pages = _pages(kv_heads=16, sequences=2000)
    for count, chosen in ((3, None), (3, PTR)):
        c = _query(heads=16, rows=100000, longest_q=100000, count=count, chosen=chosen)
        assert lib.xsv_pages_attend_workspace(C.byref(pages), C.byref(c), C.byref(nbytes)) == xsv.XSV_OK and nbytes.value == 0
    pages = _pages(kv_heads=16, sequences=1 << 24)
    assert lib.xsv_pages_attend_workspace(C.byref(pages), C.byref(c), C.byref(nbytes)) == xsv.XSV_ERR_UNSUPPORTED
    pages, c = _pages(sequences=9000000, kv_heads=1), _query(heads=1, rows=100000000, longest_q=100000000)
    assert lib.xsv_pages_attend_workspace(C.byref(pages), C.byref(c), C.byref(nbytes)) == xsv.XSV_OK
