"""Rows that are not finite, stored as 8-bit rows of pages: an infinity or NaN becomes NaN, the rest of its row stays what it is."""
import math

import pytest
import torch

from . import pages_ref as ref
from .test_gpu_pages import BF16, on_gpu, pages_of

pytestmark = pytest.mark.gpu


def spoiled(shape, g):
    """Rows of which some hold one infinity or NaN, some nothing else."""
    x = torch.randn(shape, generator=g).to(BF16)
    flat = x.view(-1, shape[-1])
    for i, bad in enumerate((math.inf, -math.inf, math.nan)):
        flat[i::7, 5 + i] = bad
    flat[3::7] = math.nan
    flat[4::7, ::2] = math.inf
    return x


def same_rows(codes, exps, x):
    """Codes and exponents of rows x, as those of the row without what is not finite, NaN there."""
    fine = torch.isfinite(x)
    want, e = ref.encode(torch.where(fine, x, torch.zeros_like(x)))
    assert bool(codes[~fine].view(torch.float8_e4m3fn).float().isnan().all())
    assert torch.equal(codes[fine], want[fine]) and torch.equal(exps, e)


@pytest.mark.parametrize("d", [64, 128])
def test_prompt(d):
    n, g = 50, torch.Generator().manual_seed(d)
    t = ref.make_pages(1, 2, d, 16, 4, BF16, 1, fp8=True)
    K, V = spoiled((1, 2, n, d), g), spoiled((1, 2, n, d), g)
    gt = on_gpu(t)
    pages_of(gt, 2).d2o_pages_fill(K.cuda(), V.cuda(), n)
    p, r = ref.entries(t, 0, n)
    for name, x in (("k", K), ("v", V)):
        same_rows(gt[name].cpu()[p, :, r], gt[name + "_exp"].cpu()[p, :, r], x[0].transpose(0, 1))


@pytest.mark.parametrize("d", [64, 128])
def test_new_tokens(d):
    """They are stored so, and reach the columns (V) and heads (K) that they belong to."""
    B, g = 14, torch.Generator().manual_seed(d)
    t = ref.make_pages(B, 2, d, 16, 4, BF16, 2, fp8=True, score=False, pos=False)
    k, v = torch.randn((B, 2, d), generator=g).to(BF16), spoiled((B, 2, d), g)
    k[3, 1, 9], k[4, 0, 0] = math.nan, math.inf
    q = torch.randn((B, 4, d), generator=g).to(BF16)
    lens = torch.arange(33, 33 + B, dtype=torch.int32)
    gt = on_gpu(t)
    out = torch.zeros((B, 4, d), dtype=BF16, device="cuda:0")
    pages_of(gt, 4).d2o_pages_step(q.cuda(), k.cuda(), v.cuda(), lens.cuda(), out)
    clean_k, clean_v = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (k, v))
    want, tol, *_ = ref.step_ref(t, q, clean_k, clean_v, lens, None, 0, 0, 64, BF16)
    out = out.cpu().double()
    bad = ~torch.isfinite(v).repeat_interleave(2, 1)
    bad[3, 2:], bad[4, :2] = True, True
    assert bool(out[bad].isnan().all()) and bool(((out - want).abs() <= tol)[~bad].all())
    for b in range(B):
        p, r = ref.entries(t, b, int(lens[b]))
        for name, x in (("k", k), ("v", v)):
            same_rows(gt[name].cpu()[p[-1], :, r[-1]], gt[name + "_exp"].cpu()[p[-1], :, r[-1]], x[b])
