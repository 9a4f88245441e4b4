"""Queries and keys that are normed before they are rotated: from the projection, which rotates by its positions, every token as a sequence of
its own at position 0, whose angle is zero; then the norms with the rotation by the tokens' positions."""
import pytest
import torch

from paper_2406_13035_amd import binding

from . import serving_ref as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.mark.parametrize("tokens,hq,hkv,hidden", [(1, 4, 2, 128), (70, 8, 2, 256), (300, 4, 4, 96)])
def test_projection_then_norms(tokens, hq, hkv, hidden):
    d, base = 128, 10000.0
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((tokens, hidden), generator=g).to(BF16)
    w = (torch.randn(((hq + 2 * hkv) * d, hidden), generator=g) / hidden ** 0.5).to(BF16)
    wq, wk = ((1 + 0.2 * torch.randn(d, generator=g)).to(BF16) for _ in range(2))
    at = torch.randint(0, 100000, (tokens,), generator=g, dtype=torch.int32)
    Q, K, V = binding.d2o_qkv_project(x.cuda()[:, None], w.cuda(), hq, hkv, d)
    plain = (x.double() @ w.double().T).view(tokens, hq + 2 * hkv, d)
    mag = (x.double().abs() @ w.double().abs().T).view(tokens, hq + 2 * hkv, d)
    got = torch.cat([Q, K, V], 1)[:, :, 0].cpu()
    # not rotated: sums of `hidden` products in fp32, rounded once
    assert bool(((got.double() - plain).abs() <= plain.abs() * 2.0 ** -8 + mag * hidden * 2.0 ** -24 + 1e-38).all())
    q, k = Q[:, :, 0].transpose(0, 1)[None], K[:, :, 0].transpose(0, 1)[None]
    binding.d2o_qk_norm_rope(q, k, wq.cuda(), wk.cuda(), positions=at.cuda()[None], rope_base=base, Q_out=q, K_out=k)
    for out, rows, weight in ((Q, got[:, :hq], wq), (K, got[:, hq:hq + hkv], wk)):
        want, tol = ref.norm_ref(rows.transpose(0, 1)[None], weight, 1e-6, d, at[None], base)
        assert bool(((out[:, :, 0].cpu().double() - want[0].transpose(0, 1)).abs() <= tol[0].transpose(0, 1)).all())
