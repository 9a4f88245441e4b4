"""Means of small values over long caches of 4-bit rows: where the bound that the calls document for them ends."""
import pytest
import torch

from . import serving_ref as ref
from .test_gpu_pages_fp4 import BF16, on_gpu, pages_of, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("signs", [False, True], ids=["positive", "both signs"])
@pytest.mark.parametrize("scale", [1e-30, 1e-33, 1e-35])
@pytest.mark.parametrize("d,n,m", [(64, 32768, 2), (64, 300, 40), (128, 5000, 3), (128, 300, 40)])
def test_means_of_small_values(d, n, m, scale, signs):
    """Sums are formed of weights times 2^-b, where 2^b is at most 512 times the entries n, and have no bits below 2^-149.  So each of n
    products and n partial sums is off by at most 2^-149, and the mean, their quotient by the sum of the weights (one over the largest probability P,
    times 2^-b, at least), by 2 n 2^-149 * 512 n P more than where numbers have no least one."""
    g = torch.Generator().manual_seed(n)
    t = ref.make_pages4(1, 1, d, 64, -(-n // 64), 3, score=False, pos=False)
    v = torch.randn(t["v"].shape[:3] + (d,), generator=g) * scale
    t["v"], t["v_exp"] = ref.encode4((v if signs else v.abs()).to(BF16))
    q = (0.3 * torch.randn((m, 2, d), generator=g)).to(BF16)
    out = torch.zeros(q.shape, dtype=BF16)
    w = ref.values(t)
    want, tol = ref.attend_ref(w, q, [0, m], [n], None, 0, 0, 1 << 20, out)
    page = t["table"][0].long()
    k = w["k"][page, 0].flatten(0, 1)[:n]
    for i in range(m):
        p = torch.softmax(q[i].double() @ k[:n - m + i + 1].T / d ** 0.5, -1)
        tol[i] += (2 * n * 2.0 ** -149 * 512 * n) * p.amax(-1, keepdim=True)
    assert bool((want.abs().amax() > 0).all())
    gt = on_gpu(t)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    og = out.cuda()
    pages_of(gt, 2).d2o_pages_attend(q.cuda(), i32([0, m]), i32([n]), og)
    within(og, want, tol)
    one = torch.zeros((1, 2, d), dtype=BF16, device="cuda:0")
    pages_of(gt, 2).d2o_pages_step(q[-1:].cuda(), None, None, i32([n]), one)
    within(one, want[-1:], tol[-1:])
