"""The workspace of attention of several tokens: one that was made for a turn of n tokens serves every smaller one."""
import ctypes as C

import pytest
import torch

from paper_2406_13035_amd import binding

from . import serving_ref as ref
from .test_gpu_pages_fp4 import BF16, on_gpu, pages_of, within
from .test_serving_host import CAPACITY, OK, PTR, lib, pages4, view  # noqa: F401

TURNS = [0, 1, 2, 3, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 200, 383, 384, 385, 500, 1000, 2047, 2048, 5000, 20000]


@pytest.mark.parametrize("batch,hq,hkv,max_len", [(2, 8, 2, 100000), (1, 32, 8, 131072), (16, 32, 8, 8192), (1, 1, 1, 2048), (64, 16, 16, 3000), (1, 500, 500, 9000), (3, 8, 8, 600)])
def test_sizes_never_fall(lib, batch, hq, hkv, max_len):  # noqa: F811
    p, v = pages4(batch=batch, n_q_heads=hq, n_kv_heads=hkv, max_pages=1 << 16), view()
    r, last = C.byref(p), 0

    def of(tokens, entries):
        n = C.c_size_t()
        assert lib.d2o_pages_attend_workspace_bytes(r, tokens, entries, C.byref(n)) == OK
        return n.value
    for tokens in TURNS:
        size = of(tokens, max_len)
        assert size >= last
        assert size >= of(tokens, max_len // 3)
        last = size
    assert of(0, max_len) == 0 and last <= 768 * 32 * (128 + 2) * 4 + 512
    # what is asked for is enough for itself: refused for one byte less only if it needs as much
    few = of(1, max_len)
    if few:
        assert lib.d2o_pages_attend(r, v, 1, PTR, PTR, None, max_len, 0, 0, v, PTR, 0, None) == CAPACITY


@pytest.mark.gpu
def test_one_workspace_for_turns_of_all_sizes():
    lib, d, n = binding.load_library(), 128, 2100  # noqa: F811
    t = ref.make_pages4(1, 2, d, 64, 33, 3, score=False, pos=False)
    gt = on_gpu(t)
    pages = pages_of(gt, 8)
    size = C.c_size_t()
    assert lib.d2o_pages_attend_workspace_bytes(pages._ref, 2000, n, C.byref(size)) == OK and size.value > 0
    ws = torch.empty(size.value, dtype=torch.uint8, device="cuda:0")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for m in (2000, 300, 40, 9, 1):
        q = torch.randn((m, 8, d), generator=torch.Generator().manual_seed(m)).to(BF16)
        qg, og = q.cuda(), torch.zeros(q.shape, dtype=BF16, device="cuda:0")
        first, lens = i32([0, m]), i32([n])
        qv, ov = pages._packed(qg, q.shape, "q"), pages._packed(og, q.shape, "out")
        assert lib.d2o_pages_attend(pages._ref, qv, m, first.data_ptr(), lens.data_ptr(), None, n, 0, 0, ov, ws.data_ptr(), size.value,
                                    torch.cuda.current_stream().cuda_stream) == OK
        torch.cuda.synchronize()
        some = sorted({0, m // 2, m - 1})
        for i in some:  # each as a turn of its own that ends there
            want, tol = ref.attend_ref(ref.values(t), q[i:i + 1], [0, 1], [n - m + i + 1], None, 0, 0, n, torch.zeros((1, 8, d)))
            within(og[i:i + 1], want, tol)
