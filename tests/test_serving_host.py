"""Refusals of the calls around steps over pages, before anything reaches a device, and their workspace sizes (no GPU needed)."""
import ctypes as C
import math

import pytest
import torch

from paper_2406_13035_amd import binding

PTR = 0x10000  # an aligned address that nobody looks behind: every call here is refused, or has nothing to do
OK, INVALID, UNSUPPORTED, CAPACITY = 0, -1, -2, -3
F32, BF16 = binding.D2O_F32, binding.D2O_BF16


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


def view(ptr=PTR, sb=1 << 16, sh=1 << 12, sn=128):
    return binding.d2o_view(ptr, sb, sh, sn)


def pages4(**kw):
    p = binding.d2o_pages(2, 8, 2, 128, BF16, 0, 16, 100, 10, view(sn=64), view(sn=64), PTR, PTR, PTR, PTR, PTR, 1)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


# ---- norms ---------------------------------------------------------------------------------

NORM = dict(batch=2, n=10, hq=8, hkv=2, d=128, dtype=BF16, Q=view(), K=view(), wq=PTR, wk=PTR, eps=1e-6, rot=128, pos=PTR, pos0=0,
            base=10000.0, Qo=view(), Ko=view())
BAD_NORM = [
    (dict(batch=0), INVALID), (dict(n=0), INVALID), (dict(hq=-1), INVALID), (dict(hkv=-1), INVALID), (dict(hq=0, hkv=0), INVALID),
    (dict(d=96), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(rot=-16), INVALID), (dict(rot=144), INVALID),
    (dict(rot=24), INVALID), (dict(eps=0.0), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=2.0), INVALID), (dict(eps=-1e-6), INVALID),
    (dict(base=1.0), INVALID), (dict(base=math.inf), INVALID), (dict(base=math.nan), INVALID), (dict(Q=view(None)), INVALID),
    (dict(K=view(PTR + 8)), INVALID), (dict(Qo=view(None)), INVALID), (dict(Ko=view(sn=130)), INVALID), (dict(Q=view(sb=-128)), INVALID),
    (dict(Qo=view(sn=64)), INVALID), (dict(Ko=view(sh=0)), INVALID), (dict(Qo=view(sb=0)), INVALID), (dict(wq=PTR + 1), INVALID),
    (dict(pos=PTR + 2), INVALID), (dict(n=1 << 28), UNSUPPORTED), (dict(hq=65530, hkv=10), UNSUPPORTED),
    (dict(dtype=F32, wk=PTR + 2), INVALID),
]


def norm(lib, **kw):
    a = {**NORM, **kw}
    return lib.d2o_qk_norm_rope(a["batch"], a["n"], a["hq"], a["hkv"], a["d"], a["dtype"], a["Q"], a["K"], a["wq"], a["wk"], a["eps"],
                                a["rot"], a["pos"], a["pos0"], a["base"], a["Qo"], a["Ko"], None)


@pytest.mark.parametrize("change,want", BAD_NORM, ids=str)
def test_norms_that_are_refused(lib, change, want):
    assert norm(lib, **change) == want


# ---- maps ----------------------------------------------------------------------------------

MAP = dict(batch=4, page=16, n_pages=100, max_pages=10, table=PTR, lens=PTR, change=PTR, ring=PTR, state=PTR, rows=64, lens_out=PTR,
           state_out=PTR, first=PTR, slots=PTR, positions=PTR, ws=None, ws_bytes=0)
BAD_MAP = [(dict([(k, 0)]), INVALID) for k in ("batch", "n_pages", "max_pages", "page")]
BAD_MAP += [(dict([(k, None)]), INVALID) for k in ("table", "lens", "change", "ring", "state", "lens_out", "state_out", "first", "slots", "positions")]
BAD_MAP += [(dict([(k, PTR + 2)]), INVALID) for k in ("table", "lens", "change", "ring", "state", "lens_out", "state_out", "first", "positions")]
BAD_MAP += [(dict(slots=PTR + 4), INVALID), (dict(page=24), INVALID), (dict(page=2048), INVALID), (dict(rows=-1), INVALID), (dict(max_pages=1 << 28), INVALID),
            (dict(rows=5000), INVALID), (dict(rows=5000, ws=PTR, ws_bytes=4), CAPACITY), (dict(batch=1025, ws=PTR + 4, ws_bytes=1 << 20), INVALID),
            (dict(batch=1 << 26, max_pages=1 << 10, ws=PTR, ws_bytes=1 << 40), UNSUPPORTED)]


@pytest.mark.parametrize("change,want", BAD_MAP, ids=str)
def test_maps_that_are_refused(lib, change, want):
    a = {**MAP, **change}
    assert lib.d2o_pages_map(a["batch"], a["page"], a["n_pages"], a["max_pages"], a["table"], a["lens"], a["change"], a["ring"], a["state"],
                             a["rows"], a["lens_out"], a["state_out"], a["first"], a["slots"], a["positions"], a["ws"], a["ws_bytes"],
                             None) == want


def test_workspaces_of_maps(lib):
    def of(batch, max_pages, rows):
        n = C.c_size_t(7)
        return lib.d2o_pages_map_workspace_bytes(batch, max_pages, rows, C.byref(n)), n.value
    assert of(64, 129, 64) == (OK, 0)
    for big in ((1025, 1, 1), (64, 129, 5000), (1000, 1000, 1)):
        rc, n = of(*big)
        assert rc == OK and n >= 4 * (4 * big[0] + 2)
    assert of(0, 1, 1)[0] == of(1, 0, 1)[0] == of(1, 1, -1)[0] == INVALID
    assert lib.d2o_pages_map_workspace_bytes(1, 1, 1, None) == INVALID


# ---- 4-bit rows ----------------------------------------------------------------------------

BAD_PAGES = [
    (dict(cache_fp4=2), INVALID), (dict(cache_fp4=-1), INVALID), (dict(cache_fp8=1), INVALID), (dict(dtype=F32), UNSUPPORTED), (dict(K_exp=None), INVALID),
    (dict(V_exp=None), INVALID), (dict(K_exp=PTR + 2), INVALID), (dict(V_exp=PTR + 1), INVALID), (dict(head_dim=32), UNSUPPORTED),
    (dict(K=view(sn=72)), INVALID), (dict(V=view(PTR + 8)), INVALID), (dict(n_q_heads=34), UNSUPPORTED),
]
ROWS_TOO_CLOSE = [dict(K=view(sn=48)), dict(V=view(sn=32)), dict(K=view(sh=16, sn=64)), dict(V=view(sb=0, sn=64))]


@pytest.mark.parametrize("change,want", BAD_PAGES, ids=str)
def test_pages_of_4_bit_rows_that_are_refused(lib, change, want):
    p, v, n = pages4(**change), view(), C.c_size_t()
    r = C.byref(p)
    assert lib.d2o_pages_workspace_bytes(r, 100, C.byref(n)) == want
    assert lib.d2o_pages_step(r, v, v, v, PTR, None, 10, 0, 0, v, PTR, 1 << 30, None) == want
    assert lib.d2o_pages_fill(r, v, v, 10, None, PTR, 5, 0, 0, PTR, 1 << 30, None) == want
    assert lib.d2o_pages_evict(r, PTR, 10, 5, 0, 0, PTR, 1 << 30, None) == want
    assert lib.d2o_pages_put(r, v, v, 10, PTR, PTR, None) == want
    assert lib.d2o_pages_get(r, v, v, 10, PTR, None) == want
    assert lib.d2o_pages_attend_workspace_bytes(r, 10, 100, C.byref(n)) == want
    assert lib.d2o_pages_attend(r, v, 10, PTR, PTR, None, 100, 0, 0, v, PTR, 1 << 30, None) == want


@pytest.mark.parametrize("change", ROWS_TOO_CLOSE, ids=str)
def test_rows_that_share_memory_are_not_written(lib, change):
    p, v = pages4(**change), view()
    r = C.byref(p)
    assert lib.d2o_pages_step(r, v, v, v, PTR, None, 10, 0, 0, v, PTR, 1 << 30, None) == INVALID
    assert lib.d2o_pages_fill(r, v, v, 10, None, PTR, 5, 0, 0, PTR, 1 << 30, None) == INVALID
    assert lib.d2o_pages_evict(r, PTR, 10, 5, 0, 0, PTR, 1 << 30, None) == INVALID
    assert lib.d2o_pages_put(r, v, v, 10, PTR, PTR, None) == INVALID


def test_rows_of_tokens_that_are_refused(lib):
    p, v = pages4(), view()
    r = C.byref(p)
    for K, V, n, slots, positions in ((view(None), v, 5, PTR, PTR), (v, view(PTR + 2), 5, PTR, PTR), (v, view(sn=4), 5, PTR, PTR), (v, v, -1, PTR, PTR),
                                      (v, v, 5, None, PTR), (v, v, 5, PTR + 4, PTR), (v, v, 5, PTR, PTR + 1), (v, v, 5, PTR, None)):
        assert lib.d2o_pages_put(r, K, V, n, slots, positions, None) == INVALID
    for K, V, n, slots in ((view(None), v, 5, PTR), (v, view(PTR + 2), 5, PTR), (v, v, -1, PTR), (v, v, 5, None), (v, v, 5, PTR + 4),
                           (view(sn=64), v, 5, PTR), (v, view(sh=0), 5, PTR)):
        assert lib.d2o_pages_get(r, K, V, n, slots, None) == INVALID
    assert lib.d2o_pages_put(r, v, v, (1 << 26) + 1, PTR, PTR, None) == UNSUPPORTED
    assert lib.d2o_pages_get(r, v, v, (1 << 26) + 1, PTR, None) == UNSUPPORTED
    assert lib.d2o_pages_put(r, v, v, 0, None, None, None) == lib.d2o_pages_get(r, v, v, 0, None, None) == OK


def test_attention_of_tokens_that_is_refused(lib):
    p, v, n = pages4(), view(), C.c_size_t()
    r = C.byref(p)

    def attend(pages=r, q=v, tokens=10, first=PTR, lens=PTR, positions=None, max_len=100, window=0, n_sink=0, out=v, ws=PTR, ws_bytes=1 << 40):
        return lib.d2o_pages_attend(pages, q, tokens, first, lens, positions, max_len, window, n_sink, out, ws, ws_bytes, None)
    for kw in (dict(q=view(None)), dict(q=view(PTR + 4)), dict(q=view(sn=4)), dict(out=view(None)), dict(out=view(sn=0)), dict(out=view(sh=64)),
               dict(tokens=-1), dict(first=None), dict(lens=None), dict(first=PTR + 2), dict(lens=PTR + 1), dict(positions=PTR + 3),
               dict(max_len=0), dict(window=-1), dict(n_sink=-1), dict(tokens=0, window=-1)):
        assert attend(**kw) == INVALID, kw
    assert attend(max_len=161) == CAPACITY
    assert attend(tokens=0, first=None, q=view(None)) == OK
    for other in (pages4(cache_fp4=0, K_exp=None, V_exp=None, K=view(), V=view()), pages4(cache_fp4=0, cache_fp8=1, K=view(), V=view())):
        assert attend(pages=C.byref(other)) == UNSUPPORTED
        assert lib.d2o_pages_attend_workspace_bytes(C.byref(other), 10, 100, C.byref(n)) == UNSUPPORTED
    assert attend(tokens=1 << 28) == UNSUPPORTED
    long = pages4(max_pages=10000)
    assert lib.d2o_pages_attend_workspace_bytes(C.byref(long), 10, 100000, C.byref(n)) == OK and n.value > 0
    assert attend(pages=C.byref(long), max_len=100000, ws_bytes=n.value - 1) == CAPACITY
    assert attend(pages=C.byref(long), max_len=100000, ws=None) == attend(pages=C.byref(long), max_len=100000, ws=PTR + 8) == INVALID
    assert lib.d2o_pages_attend_workspace_bytes(r, 0, 100, C.byref(n)) == OK and n.value == 0
    assert lib.d2o_pages_attend_workspace_bytes(r, -1, 100, C.byref(n)) == lib.d2o_pages_attend_workspace_bytes(r, 5, 0, C.byref(n)) == INVALID
    assert lib.d2o_pages_attend_workspace_bytes(r, 5, 100, None) == INVALID


# ---- the binding's own checks --------------------------------------------------------------

def test_tensors_that_are_refused():
    x = torch.zeros((1, 2, 3, 64))
    for call in (lambda: binding.d2o_qk_norm_rope(x, x), lambda: binding.d2o_qk_norm_rope(None, None),
                 lambda: binding.d2o_pages_map(torch.zeros((2, 3), dtype=torch.int32), *[torch.zeros(2, dtype=torch.int32)] * 4, 16, 8),
                 lambda: binding.Pages(torch.zeros((3, 2, 16, 32), dtype=torch.uint8), torch.zeros((3, 2, 16, 32), dtype=torch.uint8),
                                       torch.zeros((1, 3), dtype=torch.int32), 2, K_exp=torch.zeros((3, 2, 16, 2), dtype=torch.int8),
                                       V_exp=torch.zeros((3, 2, 16, 2), dtype=torch.int8))):
        with pytest.raises(binding.D2OError):
            call()
