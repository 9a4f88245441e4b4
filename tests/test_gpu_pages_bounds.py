"""Calls whose bounds are as large as they may be, on sequences that are short."""
import pytest
import torch

from . import pages_ref as ref
from .test_gpu_pages import F32, on_gpu, pages_of, same

pytestmark = pytest.mark.gpu


def test_evict_under_a_bound_of_2_to_the_28_entries():
    """More moves than a grid of a row each could hold are possible by the bound; there are none, and the call says so."""
    t = ref.make_pages(1, 1, 128, 1024, 2, F32, 1)
    table = torch.full((1, 1 << 18), -1, dtype=torch.int32)
    table[:, :2] = t["table"]
    t["table"] = table
    gt = on_gpu(t)
    pages = pages_of(gt, 1)
    pages.d2o_pages_evict(torch.tensor([1500], dtype=torch.int32, device="cuda:0"), 1 << 27, 10, 4)
    torch.cuda.synchronize()
    same(gt, t)
