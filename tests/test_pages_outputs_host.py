"""Views to be written whose rows share memory are refused before anything reaches a device (no GPU needed); views that are only read may
share theirs."""
import ctypes as C

import pytest

from .test_pages_host import CAPACITY, INVALID, PTR, lib, pages, view  # noqa: F401

SHARED = [view(sb=0), view(sh=0), view(sn=0), view(sb=120), view(sh=64), view(sn=96)]


@pytest.mark.parametrize("v", SHARED, ids=lambda v: f"{v.stride_b}-{v.stride_h}-{v.stride_n}")
def test_outputs_whose_rows_overlap(lib, v):  # noqa: F811
    ok = view()

    def window(o, q=ok, k=ok, size=1 << 30):
        return lib.d2o_window_attend(2, 50, 4, 2, 128, 1, q, k, k, None, 10, 2, o, PTR, size, None)
    assert window(v) == INVALID
    assert window(ok, v, v, 0) == CAPACITY  # (read only: refused for the workspace alone)
    for change in (dict(K=v), dict(V=v)):
        p = pages(**change)
        assert lib.d2o_pages_fill(C.byref(p), ok, ok, 10, None, PTR, 5, 0, 0, PTR, 1 << 30, None) == INVALID
        assert lib.d2o_pages_evict(C.byref(p), PTR, 10, 5, 0, 0, PTR, 1 << 30, None) == INVALID
        assert lib.d2o_pages_step(C.byref(p), ok, ok, ok, PTR, None, 10, 0, 0, ok, PTR, 1 << 30, None) == INVALID
        none = view(None)
        assert lib.d2o_pages_step(C.byref(p), ok, none, none, PTR, None, 10, 0, 0, ok, PTR, 0, None) == CAPACITY
    if v.stride_n == 128:  # (out has no rows below its heads)
        assert lib.d2o_pages_step(C.byref(pages()), ok, ok, ok, PTR, None, 10, 0, 0, v, PTR, 1 << 30, None) == INVALID


def test_a_stride_that_takes_no_part_may_be_anything(lib):  # noqa: F811
    none, one = view(None), view(sb=0, sh=0, sn=0)
    p = pages(batch=1, n_q_heads=1, n_kv_heads=1, page_size=1, n_pages=1, K=one, V=one)
    assert lib.d2o_pages_step(C.byref(p), one, none, none, PTR, None, 5, 0, 0, one, PTR, 0, None) == CAPACITY
    assert lib.d2o_window_attend(1, 1, 1, 1, 128, 1, one, one, one, None, 0, 0, one, PTR, 0, None) == CAPACITY
    assert lib.d2o_pages_fill(C.byref(p), one, one, 1, None, PTR, 5, 0, 0, PTR, 0, None) == CAPACITY
