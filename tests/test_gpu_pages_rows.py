"""Rows of single tokens into pages and out of them (d2o_pages_put, d2o_pages_get), of every format."""
import math

import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref
from . import serving_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
FORMS = ["f32", "bf16", "fp8", "fp4"]


def empty_pool(form, n_pages, Hkv, page, d, order="pool", score=True, pos=True):
    """Pool tensors on the GPU, with something in every byte."""
    dt = {"f32": F32, "bf16": BF16}.get(form, torch.uint8)
    wide = d // 2 if form == "fp4" else d
    g = torch.Generator().manual_seed(9)
    t = {}
    for x in ("k", "v"):
        raw = torch.randint(0, 120, (n_pages, Hkv, page, wide), generator=g)
        raw = raw.transpose(1, 2).contiguous().transpose(1, 2) if order == "token" else raw
        t[x] = raw.to(dt).cuda()
        t[x + "_exp"] = None
        if form in ("fp8", "fp4"):
            shape = (n_pages, Hkv, page) + ((d // 32,) if form == "fp4" else ())
            t[x + "_exp"] = torch.randint(-9, 9, shape, generator=g, dtype=torch.int8).cuda()
    t["score"] = torch.rand((n_pages, Hkv, page), generator=g).cuda() if score else None
    t["pos"] = torch.randint(0, 99, (n_pages, Hkv, page), generator=g, dtype=torch.int32).cuda() if pos else None
    t["table"] = torch.zeros((1, 1), dtype=torch.int32, device="cuda:0")
    return t


def pages_of(t, Hkv):
    return binding.Pages(t["k"], t["v"], t["table"], Hkv, K_exp=t["k_exp"], V_exp=t["v_exp"], score=t["score"], pos=t["pos"])


def held(form, x):
    """(codes or rows, powers of two, values) of rows x [.., d]."""
    if form == "fp4":
        c, e = ref.encode4(x)
        return c, e, ref.decode4(c, e)
    if form == "fp8":
        c, e = pages_ref.encode(x)
        return c, e, torch.ldexp(c.view(torch.float8_e4m3fn).double(), e.int()[..., None])
    return x, None, x.double()


def equal(a, b):
    """The same values, NaN where NaN."""
    a, b = a.double(), b.double()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def put_get(form, T, Hkv, d, page, n_pages, K, V, slots, positions, **kw):
    t = empty_pool(form, n_pages, Hkv, page, d, **kw)
    before = {k: None if x is None else x.clone() for k, x in t.items()}
    pages = pages_of(t, Hkv)
    sg = slots.cuda()
    pages.d2o_pages_put(K.cuda(), V.cuda(), sg, None if positions is None else positions.cuda())
    Ko, Vo = (torch.full((T, Hkv, d), 7.0, dtype=K.dtype, device="cuda:0") for _ in range(2))
    pages.d2o_pages_get(sg, Ko, Vo)
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < n_pages * page)
    at = (slots[ok] // page, slice(None), slots[ok] % page)
    other = torch.ones((n_pages, page), dtype=torch.bool)
    other[at[0], at[2]] = False
    for x, name, out in ((K, "k", Ko), (V, "v", Vo)):
        code, e, value = held(form, x[ok])
        assert equal(out.cpu()[ok], value.to(K.dtype)), name
        assert bool((out.cpu()[~ok] == 7).all())
        if form == "fp4":
            assert equal(ref.decode4(t[name].cpu()[at], t[name + "_exp"].cpu()[at]), value)
            assert torch.equal(t[name + "_exp"].cpu()[at], e)
        elif form == "fp8":
            assert torch.equal(t[name].cpu()[at], code) and torch.equal(t[name + "_exp"].cpu()[at], e)
        for y in (name, name + "_exp"):
            if t[y] is not None:
                assert torch.equal(t[y].cpu().transpose(1, 2)[other], before[y].cpu().transpose(1, 2)[other])
    for y, new in (("score", 0.0), ("pos", None)):
        if t[y] is not None:
            assert torch.equal(t[y].cpu().transpose(1, 2)[other], before[y].cpu().transpose(1, 2)[other])
            want = torch.zeros((int(ok.sum()), Hkv)) if y == "score" else positions[ok][:, None].expand(-1, Hkv)
            assert torch.equal(t[y].cpu()[at], want.to(t[y].dtype))
    return t


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,Hkv,page", [(1, 1, 1), (3, 2, 16), (17, 8, 64), (100, 5, 8), (333, 9, 1024), (31, 32, 2)], ids=str)
def test_put_and_get(form, d, T, Hkv, page):
    g = torch.Generator().manual_seed(T)
    n_pages = -(-2 * T // page) + 1
    dt = F32 if form == "f32" else BF16
    K, V = ((torch.randn((T, Hkv, d), generator=g) * torch.exp(torch.randn((T, Hkv, d), generator=g))).to(dt) for _ in range(2))
    slots = torch.randperm(n_pages * page, generator=g)[:T]
    if T > 2:  # tokens that have no slot
        slots[1], slots[-1] = -1, n_pages * page
    put_get(form, T, Hkv, d, page, n_pages, K, V, slots, torch.randint(0, 1 << 30, (T,), generator=g, dtype=torch.int32))


@pytest.mark.parametrize("form", FORMS)
def test_forms(form):
    g = torch.Generator().manual_seed(1)
    dt = F32 if form == "f32" else BF16
    wide = torch.randn((40, 3, 160), generator=g).to(dt)
    K, V = wide[..., 16:144], wide[..., 32:160]
    slots = torch.randperm(64, generator=g)[:40]
    put_get(form, 40, 3, 128, 16, 4, K, V, slots, None, pos=False, score=False)
    put_get(form, 40, 3, 128, 16, 4, K, V, slots, torch.arange(40, dtype=torch.int32), order="token")
    by_head = torch.randn((3, 40, 64), generator=g).to(dt).transpose(0, 1)
    put_get(form, 40, 3, 64, 16, 4, by_head, by_head, slots, torch.arange(40, dtype=torch.int32))
    put_get(form, 40, 3, 64, 16, 4, by_head, by_head, torch.full((40,), -(1 << 62)), torch.arange(40, dtype=torch.int32))


def test_every_bf16_number_as_a_block_of_its_own():
    """All finite numbers of the type, alone in their block, and as the smaller ones beside a larger one."""
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF16)
    x = x[torch.isfinite(x.float())]
    T = x.numel() // 4
    for fill in (0.0, 1.0, 3e38, 1e-30):
        K = torch.full((T, 1, 128), fill, dtype=BF16)
        K[:, 0, 5::32] = x.view(T, 4)
        put_get("fp4", T, 1, 128, 1024, -(-T // 1024), K, -K, torch.arange(T), None, pos=False, score=False)


def test_borders_between_codes():
    """Quarters of the grid's steps around every border, for several powers of two: ties go to the even code."""
    steps = torch.arange(0, 6 * 64 + 1, dtype=torch.float32) / 64.0
    rows = []
    for e in (-120, -100, -3, 0, 5, 100, 125):
        for s in (1.0, -1.0):
            block = torch.zeros((len(steps), 32))
            block[:, 0] = 6.0
            block[:, 1] = steps * s
            rows.append(block * 2.0 ** e)
    x = torch.cat(rows).to(BF16)
    x = torch.cat([x, x], -1)[:, None]
    put_get("fp4", len(x), 1, 64, 64, -(-len(x) // 64), x, x, torch.arange(len(x)), None, pos=False, score=False)


@pytest.mark.parametrize("d", [64, 128])
def test_infinities_and_nan_stay_in_their_block(d):
    g = torch.Generator().manual_seed(d)
    K = torch.randn((20, 2, d), generator=g).to(BF16)
    V = K.clone()
    K[3, 1, 40], K[4, 0, 0], V[5, 1, d - 1], V[6, 0, 31] = math.inf, -math.inf, math.nan, math.nan
    t = put_get("fp4", 20, 2, d, 16, 2, K, V, torch.arange(20), None, pos=False, score=False)
    for x, broken in (("k", 2), ("v", 2)):
        assert int((t[x + "_exp"].cpu().transpose(1, 2).flatten(0, 1)[:20] == -128).sum()) == broken
