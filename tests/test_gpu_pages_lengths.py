"""Attention of several tokens per sequence where lengths are zero, negative or larger than the bound."""
import pytest
import torch

from . import serving_ref as ref
from .test_gpu_pages_fp4 import BF16, attend_case, bits_same, on_gpu, pages_of, within

pytestmark = pytest.mark.gpu
LOW, HIGH = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("heads,news", [((1, 1), 64), ((8, 2), 33), ((4, 1), 300)], ids=str)
@pytest.mark.parametrize("window,n_sink", [(0, 0), (7, 3)])
def test_lengths_below_zero_have_no_entries(heads, news, window, n_sink):
    """Their tokens get zeros, like those of a sequence of length zero; the sequences beside them are as ever."""
    lens = [LOW, 50, -1, LOW + 20, 0, LOW + news, 70]
    attend_case(128, *heads, 16, lens, [news, 20, news, news, news, news, 70], window, n_sink)


@pytest.mark.parametrize("d", [64, 128])
def test_lengths_of_any_value(d):
    lens, news, max_len = [HIGH, LOW, 100, 90], [70, 40, 100, 3], 100
    first = [sum(news[:b]) for b in range(5)]
    t = ref.make_pages4(4, 2, d, 16, 7, 3, score=False, pos=False)
    q = torch.randn((first[-1], 4, d), generator=torch.Generator().manual_seed(1)).to(BF16)
    out = torch.full(q.shape, 7.0, dtype=BF16)
    want, tol = ref.attend_ref(ref.values(t), q, first, lens, None, 0, 0, max_len, out)
    gt, og = on_gpu(t), out.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    pages_of(gt, 4, max_len).d2o_pages_attend(q.cuda(), i32(first), i32(lens), og)
    within(og, want, tol)
    bits_same(gt, t)


@pytest.mark.parametrize("n_sink", [HIGH, HIGH - 31, HIGH - 32])
def test_as_many_first_tokens_as_there_are_numbers(n_sink):
    """A window beside first tokens without end hides nothing."""
    attend_case(128, 8, 2, 64, [5000, 40], [40, 3], window=9, n_sink=n_sink)
