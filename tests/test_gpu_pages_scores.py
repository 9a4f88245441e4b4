"""Generation steps over pages: scores beside logits that are not finite, and values near the largest number."""
import math

import pytest
import torch

from . import pages_ref as ref
from .test_gpu_pages import BF16, F32, FORMS, cuda, on_gpu, pages_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["key", "query", "infinite key", "beside minus infinity"])
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
@pytest.mark.parametrize("heads,n", [((2, 2), 100), ((8, 2), 75), ((12, 2), 101), ((2, 1), 3001), ((8, 2), 2500), ((16, 1), 3100)], ids=str)
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_scores_of_entries_that_are_not_seen_stay(dtype, heads, n, pos, what):
    """A seen logit that is NaN or infinite makes the scores of the entries that its head sees NaN, and leaves all others as they were."""
    Hq, Hkv = heads
    window, n_sink = n // 3, 5
    t = ref.make_pages(1, Hkv, 64, 16, n // 16 + 2, dtype, n, pos=pos)
    g = torch.Generator().manual_seed(n)
    q = torch.randn((1, Hq, 64), generator=g).to(dtype)
    p, r = ref.entries(t, 0, n)
    at = torch.arange(n)
    if pos:
        at = torch.randperm(n, generator=g)
        t["pos"][p, :, r] = at[:, None].to(torch.int32).expand(-1, Hkv).contiguous()
    seen = (at > n - 1 - window) | (at < n_sink)
    some = int(seen.nonzero()[7])
    head = 0 if what == "query" else Hkv - 1  # whose scores become NaN
    if what == "query":
        q[0, 0] = math.nan
    else:
        t["k"][p[some], head, r[some]] = math.inf if what == "infinite key" else math.nan
    if what == "infinite key":
        q[0, head * (Hq // Hkv):] = q[0, head * (Hq // Hkv):].abs()
    if what == "beside minus infinity":
        other = int(seen.nonzero()[12])
        t["k"][p[other], head, r[other]] = -math.inf
        q[0, head * (Hq // Hkv):] = q[0, head * (Hq // Hkv):].abs()
    gt = on_gpu(t)
    out = torch.zeros((1, Hq, 64), dtype=dtype, device="cuda:0")
    last = torch.tensor([n - 1], dtype=torch.int32)
    pages_of(gt, Hq).d2o_pages_step(q.cuda(), None, None, *cuda(torch.tensor([n], dtype=torch.int32)), out, positions=last.cuda(),
                                    window=window, n_sink=n_sink)
    got, was = gt["score"].cpu(), t["score"]
    touched = torch.zeros(was.shape, dtype=torch.bool)
    for h in range(Hkv):
        touched[p[seen], h, r[seen]] = True
        now = got[p[seen], h, r[seen]]
        assert bool(now.isnan().all()) if h == head else bool(torch.isfinite(now).all() and (now >= was[p[seen], h, r[seen]]).all())
    assert torch.equal(got[~touched], was[~touched])


@pytest.mark.parametrize("heads,n", [((1, 1), 2), ((2, 2), 700), ((4, 1), 5000), ((8, 1), 700), ((16, 1), 9001), ((4, 2), 20011)], ids=str)
@pytest.mark.parametrize("flat", [True, False], ids=["equal", "random"])
@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_values_near_the_largest_number(dtype, fp8, flat, heads, n):
    """A mean is no larger than what it is taken of, however many entries there are; outputs and scores within their bounds."""
    Hq, Hkv, d = *heads, 64
    t = ref.make_pages(1, Hkv, d, 16, n // 16 + 1, dtype, n, fp8, pos=False)
    big = torch.full(t["v"].shape, 2.9e38)
    big[..., ::2] = -2.9e38
    if fp8:
        t["v"], t["v_exp"] = ref.encode(big.to(BF16))
    else:
        t["v"] = big.to(dtype)
    q = (torch.randn((1, Hq, d), generator=torch.Generator().manual_seed(n)) * (0.0 if flat else 1.5)).to(dtype)
    lens = torch.tensor([n], dtype=torch.int32)
    want, tol, new, add, add_tol = ref.step_ref(t, q, None, None, lens, None, 0, 0, n, dtype)
    gt = on_gpu(t)
    out = torch.zeros((1, Hq, d), dtype=dtype, device="cuda:0")
    pages_of(gt, Hq).d2o_pages_step(q.cuda(), None, None, lens.cuda(), out)
    err = (out.cpu().double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    err = (gt["score"].cpu().double() - new["score"].double() - add).abs()
    assert bool((err <= add_tol).all()), float((err / add_tol).max())
