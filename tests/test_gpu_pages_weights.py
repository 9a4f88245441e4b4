"""How exact the weights of a step over 4-bit rows are."""
import math

import pytest
import torch

from . import serving_ref as ref
from .test_gpu_pages_fp4 import BF16, on_gpu, pages_of, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,Hkv,B", [(1, 8, 60), (3, 8, 30), (5, 8, 20), (6, 8, 20), (8, 8, 20), (9, 4, 30), (16, 4, 20)])
@pytest.mark.parametrize("score", [False, True], ids=["alone", "scores"])
def test_weights_hold_24_bits(d, G, Hkv, B, score):
    """Two entries of nearly the same weight and opposite values, beside one of value zero and a larger weight: what is left of the mean is as
    small as the weights' errors.  The logits are exact.  An exponent is rounded as a product (of a magnitude below 4: 2^-23, and 2^-22 for the
    two roundings of its factor), less the largest (2^-23 at most) and less the bias of 10 (between 8 and 16: 2^-21): below 2^-20 in all;
    times ln 2, and an ulp (2^-23) of the exponential: a weight is off by E = 2^-20 of itself at most.  The two weights p and p' of a sum S move the mean by
    E (p + p') / S, where p, p' <= S / 3.5 as the third is more than 1.5 times as large; four sums of 2^-24 beside that, and the output's rounding."""
    g = torch.Generator().manual_seed(G)
    t = ref.make_pages4(B, Hkv, d, 16, 1, 3, score=score, pos=False)
    k = torch.zeros((t["k"].shape[0], Hkv, 16, d))
    k[..., 31::32] = 6.0  # (every block's power of two is one)
    k[:, :, 1, 1], k[:, :, 2, 2] = 0.5, 1.0
    v = torch.zeros_like(k)
    v[:, :, 0], v[:, :, 1] = 1.0, -1.0
    (t["k"], t["k_exp"]), (t["v"], t["v_exp"]) = ref.encode4(k), ref.encode4(v)
    q = torch.zeros((B, Hkv * G, d))
    q[..., 1] = 2.0 ** -9
    q[..., 2] = (0.45 + 0.6 * torch.rand((B, Hkv * G), generator=g)) * math.sqrt(d)  # exp of 0.45 and more: p <= S / 3.5
    q = q.to(BF16)
    logits = q.double() @ k[0, 0, :3].double().T / math.sqrt(d)
    p = torch.softmax(logits, -1)
    want = (p[..., 0] - p[..., 1])[..., None].expand(-1, -1, d)
    tol = (2.0 ** -20 * 2 / 3.5 + 4 * 2.0 ** -24) + want.abs() * 2.0 ** -8
    gt = on_gpu(t)
    out = torch.zeros(q.shape, dtype=BF16, device="cuda:0")
    lens = torch.full((B,), 3, dtype=torch.int32, device="cuda:0")
    pages_of(gt, Hkv * G).d2o_pages_step(q.cuda(), None, None, lens, out)
    within(out, want, tol)
