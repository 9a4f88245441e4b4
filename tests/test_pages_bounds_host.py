"""Bounds whose launches would not fit a grid are refused before anything is stored (no GPU needed)."""
import ctypes as C

from .test_pages_host import PTR, UNSUPPORTED, lib, pages, view  # noqa: F401


def test_steps_whose_scores_do_not_fit_a_grid(lib):  # noqa: F811
    """Where heads are split, a workgroup of 256 threads per 1024 entries of every head, and one per query head: below 2^32 threads."""
    for batch, kv, max_len in ((256, 2, 1 << 25), (64, 2, 1 << 27), (2, 8, 0x7FFF0000)):
        p = pages(batch=batch, n_kv_heads=kv, max_pages=max_len // 16)
        v = view()
        assert lib.d2o_pages_step(C.byref(p), v, v, v, PTR, None, max_len, 0, 0, v, PTR, 1 << 62, None) == UNSUPPORTED
