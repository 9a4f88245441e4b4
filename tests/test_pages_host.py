"""Refusals of the calls on caches in pages and of windowed attention, before anything reaches a device, and their
workspace sizes (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref as ref

PTR = 0x10000  # an aligned address that nobody looks behind: every call here is refused
OK, INVALID, UNSUPPORTED, CAPACITY = 0, -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def view(ptr=PTR, sb=1 << 16, sh=1 << 12, sn=128):
    return binding.d2o_view(ptr, sb, sh, sn)


def pages(**kw):
    p = binding.d2o_pages(2, 8, 2, 128, binding.D2O_BF16, 0, 16, 100, 10, view(), view(), None, None, PTR, PTR, PTR)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def bytes_of(lib, p, max_len=100):
    n = C.c_size_t()
    return lib.d2o_pages_workspace_bytes(C.byref(p), max_len, C.byref(n)), n.value


BAD_PAGES = [
    (dict(batch=0), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_q_heads=7), INVALID), (dict(n_kv_heads=0), INVALID),
    (dict(n_q_heads=34), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(cache_fp8=2), INVALID), (dict(cache_fp8=1), INVALID), (dict(cache_fp8=1, dtype=0, K_exp=PTR, V_exp=PTR), UNSUPPORTED),
    (dict(page_size=0), INVALID), (dict(page_size=24), INVALID), (dict(page_size=2048), INVALID), (dict(n_pages=0), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=1 << 28), INVALID), (dict(page_table=None), INVALID), (dict(page_table=PTR + 2), INVALID),
    (dict(score=PTR + 1), INVALID), (dict(K=view(None)), INVALID), (dict(V=view(PTR + 8)), INVALID), (dict(K=view(sn=130)), INVALID),
    (dict(V=view(sh=4)), INVALID), (dict(K=view(sb=-128)), INVALID),
]


@pytest.mark.parametrize("change,want", BAD_PAGES, ids=str)
def test_descriptions_that_are_refused(lib, change, want):
    p = pages(**change)
    assert bytes_of(lib, p)[0] == want
    v = view()
    assert lib.d2o_pages_step(C.byref(p), v, v, v, PTR, None, 10, 0, 0, v, PTR, 1 << 30, None) == want
    assert lib.d2o_pages_fill(C.byref(p), v, v, 10, None, PTR, 5, 0, 0, PTR, 1 << 30, None) == want
    assert lib.d2o_pages_evict(C.byref(p), PTR, 10, 5, 0, 0, PTR, 1 << 30, None) == want


def test_null_and_sizes(lib):
    n = C.c_size_t()
    assert lib.d2o_pages_workspace_bytes(None, 10, C.byref(n)) == INVALID
    assert lib.d2o_pages_workspace_bytes(C.byref(pages()), 0, C.byref(n)) == INVALID
    assert lib.d2o_pages_workspace_bytes(C.byref(pages()), 10, None) == INVALID
    assert bytes_of(lib, pages(), 100)[0] == OK and bytes_of(lib, pages(), 100)[1] >= 256
    assert bytes_of(lib, pages(), 100000)[1] > bytes_of(lib, pages(), 100)[1]
    assert bytes_of(lib, pages(n_q_heads=32))[0] == OK and bytes_of(lib, pages(cache_fp8=1, K_exp=PTR, V_exp=PTR))[0] == OK


def test_step_refusals(lib):
    p, v = pages(), view()
    none = view(None)

    def call(q=v, kn=v, vn=v, lens=PTR, pos=None, max_len=100, window=0, sink=0, out=v, ws=PTR, size=1 << 30):
        return lib.d2o_pages_step(C.byref(p), q, kn, vn, lens, pos, max_len, window, sink, out, ws, size, None)
    assert call(q=none) == INVALID and call(out=none) == INVALID and call(kn=none) == INVALID and call(vn=none) == INVALID
    assert call(lens=None) == INVALID and call(max_len=0) == INVALID and call(window=-1) == INVALID and call(sink=-1) == INVALID
    assert call(q=view(PTR + 2)) == INVALID and call(out=view(sh=100)) == INVALID and call(kn=view(sb=-8)) == INVALID
    assert call(ws=None) == INVALID and call(ws=PTR + 4) == INVALID
    assert call(max_len=161) == CAPACITY and call(size=16) == CAPACITY


def test_fill_refusals(lib):
    v = view()

    def call(p=pages(), k=v, vv=v, n=100, lens=None, scores=PTR, budget=50, recent=10, sink=4, ws=PTR, size=1 << 30):
        return lib.d2o_pages_fill(C.byref(p), k, vv, n, lens, scores, budget, recent, sink, ws, size, None)
    assert call(n=0) == INVALID and call(budget=0) == INVALID and call(recent=-1) == INVALID and call(sink=-1) == INVALID
    assert call(recent=47) == INVALID and call(recent=0x7FFFFFFF, sink=0x7FFFFFFF) == INVALID
    assert call(scores=None) == INVALID and call(k=view(None)) == INVALID and call(vv=view(sn=3)) == INVALID
    assert call(ws=None) == INVALID and call(size=8) == CAPACITY and call(n=1000, budget=161) == CAPACITY


def test_evict_refusals(lib):
    def call(p=pages(), lens=PTR, max_len=100, budget=50, recent=10, sink=4, ws=PTR, size=1 << 30):
        return lib.d2o_pages_evict(C.byref(p), lens, max_len, budget, recent, sink, ws, size, None)
    assert call(lens=None) == INVALID and call(max_len=0) == INVALID and call(budget=0) == INVALID
    assert call(recent=-1) == INVALID and call(sink=-1) == INVALID and call(recent=47) == INVALID
    assert call(p=pages(score=None)) == INVALID and call(p=pages(pos=None)) == INVALID
    assert call(max_len=161) == CAPACITY and call(size=8) == CAPACITY and call(ws=PTR + 8) == INVALID
    assert call(max_len=50) == OK  # nothing can be over the budget: nothing is launched


def test_window_refusals(lib):
    v, n = view(), C.c_size_t()

    def call(B=2, n=50, hq=4, hkv=2, d=128, dt=1, q=v, k=v, vv=v, window=10, sink=2, o=v, ws=PTR, size=1 << 30):
        return lib.d2o_window_attend(B, n, hq, hkv, d, dt, q, k, vv, None, window, sink, o, ws, size, None)
    assert call(B=0) == INVALID and call(n=0) == INVALID and call(hq=3) == INVALID and call(hq=0) == INVALID and call(hkv=0) == INVALID
    assert call(d=96) == UNSUPPORTED and call(dt=7) == UNSUPPORTED and call(window=-1) == INVALID and call(sink=-1) == INVALID
    assert call(q=view(None)) == INVALID and call(o=view(PTR + 4)) == INVALID and call(k=view(sn=132)) == INVALID
    assert call(ws=None) == INVALID and call(size=0) == CAPACITY
    assert lib.d2o_window_workspace_bytes(1, 10, 1, 128, 1, None) == INVALID
    assert lib.d2o_window_workspace_bytes(1, 10, 1, 80, 1, C.byref(n)) == UNSUPPORTED
    assert lib.d2o_window_workspace_bytes(1, 10, 1, 128, 1, C.byref(n)) == OK and n.value > 0


def test_the_reference_forms_agree_with_themselves():
    """The 64-bit forms on small inputs against a transcription by hand."""
    q, k, v = (torch.randn((5, 4), dtype=torch.float64, generator=torch.Generator().manual_seed(i)) for i in range(3))
    seen = ref.window_seen(5, 2, 1)
    assert seen.tolist() == [[True, False, False, False, False], [True, True, False, False, False], [True, True, True, False, False],
                             [True, False, True, True, False], [True, False, False, True, True]]
    o, p = ref.attend64(q, k, v, seen)
    w = [math.exp(float(q[4] @ k[j]) / 2) for j in (0, 3, 4)]
    want = sum(x * v[j] for x, j in zip(w, (0, 3, 4))) / sum(w)
    assert torch.allclose(o[4], want, atol=1e-14)
    v[1] = math.inf  # rows 3 and 4 do not see it
    o2, _ = ref.attend64(q, k, v, seen)
    assert torch.allclose(o2[4], want, atol=1e-14) and bool(o2[1].isinf().all())
    order = ref.score_order(torch.tensor([1.0, math.nan, 3.0, 3.0, 0.0, 9.0]).numpy(), [5, 4, 3, 2, 1, 0],
                            [False, False, False, False, True, False], [True] * 5 + [False])
    assert order.tolist() == [4, 1, 3, 2, 0, 5]
