"""How exact the rotation's sines and cosines are."""
import pytest
import torch

from paper_2406_13035_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("far", [7, 1000, 1 << 20])
def test_sines_and_cosines_hold_24_bits(d, far):
    """Rows of ones have norm one (their sum and its root are exact, eps does not reach one's last bit), and with a weight of zero in the second
    element of each pair the results are the cosine and the sine themselves.  Each is the sine or cosine of an angle rounded to fp32, within one of fp32's
    steps (2^-24 below one), plus what the rounding of the angle took away, which is added with half a step more.  A position's product with a 64-bit factor is
    off by 2^-52 of itself, a fraction of a turn is 2 pi as much in radians."""
    n, h = 4096, d // 2
    g = torch.Generator().manual_seed(far)
    at = torch.randint(-far, far + 1, (1, n), generator=g, dtype=torch.int64).to(torch.int32)
    x = torch.ones((1, 2, n, d), device="cuda:0")
    w = torch.cat([torch.ones(h), torch.zeros(h)]).cuda()
    y, _ = binding.d2o_qk_norm_rope(x, None, w, eps=1e-20, positions=at.cuda())
    c = torch.arange(h, dtype=torch.float64)
    turns = at.double()[0, :, None] * 10000.0 ** (-2.0 * c / d)
    want = torch.cat([turns.cos(), turns.sin()], -1)
    err = (y.cpu().double() - want).abs()
    assert float(err.max()) <= 1.5 * 2.0 ** -24 + far * 2.0 ** -50, float(err.max() * 2.0 ** 24)
