"""Caches in pages whose rows are held in 4 bits: steps, prompts into them, evictions, and attention of several tokens per
sequence, against their 64-bit forms."""
import math

import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref
from . import serving_ref as ref

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def on_gpu(t):
    out = {}
    for name, x in t.items():
        out[name] = None if x is None else torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda:0").copy_(x)
    return out


def pages_of(t, q_heads, max_len=None):
    return binding.Pages(t["k"], t["v"], t["table"], q_heads, K_exp=t["k_exp"], V_exp=t["v_exp"], score=t["score"],
                         pos=t["pos"], max_len=max_len)


def cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


def within(got, want, tol):
    got = got.cpu().double()
    assert torch.equal(got.isnan(), want.isnan())
    fine = ~want.isnan()
    err = (got - want).abs()[fine]
    assert bool((err <= tol[fine]).all()), float((err / tol[fine]).max())


def same_values(gt, new):
    """Rows of the pool `gt` against values (rounding had one way to go), positions exactly."""
    for x in ("k", "v"):
        g, w = ref.decode4(gt[x].cpu(), gt[x + "_exp"].cpu()), new[x]
        assert bool(((g == w) | (g.isnan() & w.isnan())).all()), x
    if new["pos"] is not None:
        assert torch.equal(gt["pos"].cpu(), new["pos"])


# ---- one token per sequence ----------------------------------------------------------------

def step_case(d, B, Hq, Hkv, page, lens, window=0, n_sink=0, score=True, pos=False, append=True, order="pool", seed=0, max_len=None,
              spoil=None, qscale=1.5, positions=None, scale=1.0):
    lens = torch.tensor(lens, dtype=torch.int32)
    cap = -(-max(1, int(lens.max())) // page) + 1
    t = ref.make_pages4(B, Hkv, d, page, cap, seed, order, score, pos, scale=scale)
    g = torch.Generator().manual_seed(77 + seed)
    q = (torch.randn((B, Hq, d), generator=g) * qscale).to(BF16)
    kn, vn = ((torch.randn((B, Hkv, d), generator=g) * scale).to(BF16) if append else None for _ in range(2))
    if pos:  # entries in any order, with gaps
        for b in range(B):
            n = int(lens[b])
            p, r = pages_ref.entries(t, b, n)
            for h in range(Hkv):
                t["pos"][p, h, r] = (3 * torch.randperm(n, generator=g)).to(torch.int32) if n else t["pos"][p, h, r]
        if positions is None:
            positions = torch.tensor([3 * max(0, int(n) - 1) + 2 for n in lens], dtype=torch.int32)
    if spoil:
        spoil(t, lens)
    m = max_len or cap * page
    want, tol, new, add, add_tol = ref.step_ref4(t, q, kn, vn, lens, positions, window, n_sink, m)
    gt = on_gpu(t)
    pages = pages_of(gt, Hq, m)
    out = torch.full((B, Hq, d), 7.0, dtype=BF16, device="cuda:0")
    pages.d2o_pages_step(*cuda(q, kn, vn, lens), out, positions=None if positions is None else positions.cuda(), window=window,
                         n_sink=n_sink)
    torch.cuda.synchronize()
    within(out, want, tol)
    same_values(gt, new)
    if score:
        g64, w64 = gt["score"].cpu().double(), new["score"].double() + add
        untouched = add_tol == 0
        assert torch.equal(gt["score"].cpu()[untouched], new["score"][untouched])
        e = (g64 - w64).abs()[~untouched]
        assert bool((e <= add_tol[~untouched]).all()), float((e / add_tol[~untouched]).max())
    return gt


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,page,lens", [
    ((1, 1), 16, [1]), ((2, 1), 1, [2, 1]), ((4, 4), 8, [15, 16, 17]), ((3, 1), 16, [31, 33]), ((8, 1), 64, [63, 64, 65]),
    ((16, 1), 32, [100]), ((10, 2), 128, [127, 129]), ((4, 1), 256, [255, 257, 1]), ((6, 2), 2, [511, 7]),
    ((8, 8), 1024, [1025, 3]), ((2, 2), 64, [2050]), ((4, 2), 16, [700, 0, 5, 1300]), ((11, 1), 4, [77]),
], ids=str)
def test_step(d, heads, page, lens):
    step_case(d, len(lens), heads[0], heads[1], page, lens, seed=sum(lens))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
@pytest.mark.parametrize("window,n_sink,lens", [
    (1, 0, [1, 200]), (16, 4, [500, 17]), (100, 0, [100, 101]), (64, 130, [400, 60]), (1000, 1, [1500, 90]), (3, 3, [6, 7]),
], ids=str)
def test_step_through_a_window(d, pos, window, n_sink, lens):
    step_case(d, len(lens), 4, 2, 16, lens, window, n_sink, pos=pos, seed=window)
    step_case(d, len(lens), 4, 2, 4, lens, window, n_sink, pos=pos, seed=window)


def test_step_without_a_new_token_and_without_scores():
    step_case(128, 2, 8, 2, 32, [300, 41], append=False, score=False)
    step_case(64, 2, 8, 2, 32, [300, 41], append=False, score=True)
    step_case(64, 2, 8, 2, 32, [300, 41], append=True, score=False)


@pytest.mark.parametrize("heads,n", [((4, 1), 20011), ((32, 8), 9001), ((8, 8), 12288), ((16, 1), 16385)], ids=str)
def test_step_over_a_long_cache(heads, n):
    step_case(128, 1, heads[0], heads[1], 64, [n], seed=n)


def test_step_of_many_short_sequences():
    lens = [1 + (i * 37) % 90 for i in range(70)]
    step_case(64, len(lens), 4, 2, 16, lens)


@pytest.mark.parametrize("d", [64, 128])
def test_step_with_pages_whose_rows_lie_by_token(d):
    step_case(d, 2, 4, 2, 16, [100, 37], order="token")


@pytest.mark.parametrize("scale", [1e-30, 1e30, 8e36])
def test_step_with_values_of_any_size(scale):
    """Means of values near the largest number do not overflow, nor do small ones vanish.  (Keys of that size: queries of the inverse.)"""
    step_case(128, 2, 4, 2, 16, [700, 41], score=False, scale=scale, qscale=1.0 / scale)


def spoil_hidden(t, lens):
    """Rows behind the last entry hold NaN, infinite values and powers of two of any size."""
    page = t["k"].shape[2]
    for b, n in enumerate(lens.tolist()):
        for s in range(n, t["table"].shape[1] * page):
            p = int(t["table"][b, s // page])
            t["k_exp"][p, :, s % page] = -128 if s % 2 else 127
            t["v_exp"][p, :, s % page] = -128 if s % 3 else 127


@pytest.mark.parametrize("page", [4, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_step_beside_rows_of_nan_behind_the_end(d, page):
    step_case(d, 3, 4, 2, page, [70, 33, 16], spoil=spoil_hidden)


@pytest.mark.parametrize("page", [4, 64])
def test_step_beside_hidden_and_missing_entries_of_nan(page):
    def spoil(t, lens):
        spoil_hidden(t, lens)
        for b, n in enumerate(lens.tolist()):
            for s in range(8, n - 20):  # hidden by the window
                p = int(t["table"][b, s // page])
                t["v_exp"][p, :, s % page] = -128
                if s % 2:
                    t["k_exp"][p, :, s % page] = -128
    step_case(128, 2, 4, 2, page, [100, 61], window=20, n_sink=8, spoil=spoil)

    def no_page(t, lens):
        t["table"][0, 1] = -1
        t["table"][1, 0] = t["k"].shape[0]
        t["v_exp"][0] = -128  # the pool's first page, which stands for none
    step_case(128, 2, 4, 2, page, [3 * page + 1, 2 * page], spoil=no_page, append=False)


def test_nan_of_a_block_reaches_its_elements():
    def spoil(t, lens):
        p = int(t["table"][0, 1])
        t["v_exp"][p, 1, 3, 2] = -128
    gt = step_case(128, 1, 8, 2, 64, [130], spoil=spoil, score=False)
    assert int((gt["v_exp"] == -128).sum()) == 1


# ---- prompts and evictions -----------------------------------------------------------------

def bits_same(gt, want, names=("k", "v", "k_exp", "v_exp", "score", "pos")):
    for x in names:
        if want[x] is not None:
            assert torch.equal(gt[x].cpu(), want[x]), x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,budget,recent,n_sink,page", [(1, 1, 0, 0, 1), (40, 40, 3, 1, 16), (300, 57, 11, 4, 8), (5000, 700, 100, 4, 64),
                                                        (20000, 900, 200, 2, 128)], ids=str)
def test_fill(d, n, budget, recent, n_sink, page):
    B, Hkv = 2, 2
    g = torch.Generator().manual_seed(n)
    K, V = (torch.randn((B, Hkv, n, d), generator=g).to(BF16) for _ in range(2))
    scores = torch.rand((B, Hkv, n), generator=g)
    lens = torch.tensor([n, max(1, n - 7)], dtype=torch.int32)
    t = ref.make_pages4(B, Hkv, d, page, -(-budget // page), 3)
    w = ref.values(t)
    want = pages_ref.fill_ref(w, ref.rounded4(K), ref.rounded4(V), lens.tolist(), scores, budget, recent, n_sink)
    gt = on_gpu(t)
    pages_of(gt, 2, max_len=n).d2o_pages_fill(*cuda(K, V), budget, recent, n_sink, *cuda(scores, lens))
    torch.cuda.synchronize()
    same_values(gt, want)
    assert torch.equal(gt["score"].cpu(), want["score"])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 64])
@pytest.mark.parametrize("lens,budget,recent,n_sink", [([9, 8], 8, 2, 1), ([300, 100], 77, 20, 4), ([2304, 2100], 1100, 300, 4),
                                                       ([18000, 17000], 16990, 100, 0), ([20000, 19995], 19990, 100, 2)], ids=str)
def test_evict(d, page, lens, budget, recent, n_sink):
    if page == 1 and lens[0] > 10000:
        lens = [n // 50 for n in lens]
        budget, recent = budget // 50, recent // 50
    t = ref.make_pages4(2, 2, d, page, -(-max(lens) // page), 5)
    g = torch.Generator().manual_seed(1)
    for b in range(2):
        p, r = pages_ref.entries(t, b, lens[b])
        for h in range(2):
            t["pos"][p, h, r] = torch.randperm(lens[b], generator=g).to(torch.int32)
    want = pages_ref.evict_ref(t, lens, budget, recent, n_sink)
    gt = on_gpu(t)
    pages_of(gt, 2, max_len=max(lens)).d2o_pages_evict(torch.tensor(lens, dtype=torch.int32).cuda(), budget, recent, n_sink)
    torch.cuda.synchronize()
    bits_same(gt, want)


# ---- several tokens per sequence -----------------------------------------------------------

def attend_case(d, Hq, Hkv, page, lens, news, window=0, n_sink=0, pos=False, given=False, order="pool", seed=0, max_len=None, spoil=None,
                extra=0, scale=1.0, qscale=1.5, in_place=False, first=None, score=False):
    B = len(lens)
    cap = -(-max(1, *lens) // page) + 1
    t = ref.make_pages4(B, Hkv, d, page, cap, seed, order, score, pos, scale=scale)
    g = torch.Generator().manual_seed(33 + seed)
    T = sum(news) + extra
    first = [sum(news[:b]) for b in range(B + 1)] if first is None else first
    wide = (torch.randn((T, Hq, d), generator=g) * qscale).to(BF16)
    positions = None
    if pos:
        for b in range(B):
            p, r = pages_ref.entries(t, b, lens[b])
            for h in range(Hkv):
                t["pos"][p, h, r] = (3 * torch.randperm(lens[b], generator=g)).to(torch.int32)
    if pos or given:
        positions = torch.randint(0, 3 * max(1, *lens) + 3, (T,), generator=g, dtype=torch.int32)
    if spoil:
        spoil(t, lens)
    m = max_len or cap * page
    out = torch.full((T, Hq, d), 7.0, dtype=BF16)
    if in_place:
        out = wide.clone()
    want, tol = ref.attend_ref(ref.values(t), wide, first, lens, positions, window, n_sink, m, out)
    gt = on_gpu(t)
    pages = pages_of(gt, Hq, m)
    og = out.cuda()
    qg = og if in_place else wide.cuda()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    pages.d2o_pages_attend(qg, i32(first), i32(lens), og, positions=None if positions is None else positions.cuda(), window=window,
                           n_sink=n_sink)
    torch.cuda.synchronize()
    within(og, want, tol)
    bits_same(gt, t)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,page,lens,news", [
    ((1, 1), 16, [1], [1]), ((2, 1), 1, [9], [9]), ((4, 4), 8, [15, 16, 17], [3, 1, 17]), ((3, 1), 16, [31, 33], [7, 2]),
    ((8, 1), 64, [63, 64, 65], [1, 64, 0]), ((16, 1), 32, [100], [33]), ((10, 2), 128, [127, 129], [5, 129]),
    ((8, 2), 256, [700, 0, 5, 300], [40, 0, 5, 1]), ((5, 1), 2, [77], [20]), ((4, 1), 1024, [1500, 40], [200, 40]),
    ((4, 1), 16, [900], [300]), ((8, 2), 64, [1000], [131]), ((2, 2), 32, [600, 512], [260, 256]),
], ids=str)
def test_attend(d, heads, page, lens, news):
    attend_case(d, heads[0], heads[1], page, lens, news, seed=sum(lens))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
@pytest.mark.parametrize("window,n_sink,lens,news", [
    (1, 0, [1, 200], [1, 9]), (16, 4, [300, 17], [50, 17]), (100, 0, [100, 101], [2, 101]), (64, 130, [400, 60], [90, 3]), (3, 3, [6, 7], [6, 7]),
    (200, 1, [700, 650], [170, 1]),
], ids=str)
def test_attend_through_a_window(d, pos, window, n_sink, lens, news):
    attend_case(d, 4, 2, 16, lens, news, window, n_sink, pos=pos, seed=window)
    attend_case(d, 4, 2, 4, lens, news, window, n_sink, pos=pos, seed=window)


def test_attend_forms():
    attend_case(128, 4, 2, 16, [100, 37], [5, 7], order="token")
    attend_case(128, 4, 2, 16, [100, 37], [50, 7], window=20, n_sink=3, given=True)
    attend_case(128, 4, 2, 16, [100, 37], [50, 7], extra=9)                     # rows that belong to no sequence
    attend_case(128, 4, 2, 16, [100, 37], [50, 7], in_place=True)
    attend_case(64, 4, 2, 16, [3000, 37], [150, 7], in_place=True)
    attend_case(128, 4, 2, 16, [5, 37], [9, 7])                                 # more tokens than entries
    attend_case(128, 4, 2, 16, [100, 90], [5, 60], max_len=80)                  # lengths are cut
    attend_case(128, 4, 2, 16, [100, 37, 50], [5, 7, 3], first=[-4, 9, 9, 99])  # offsets outside
    attend_case(128, 4, 2, 16, [100, 37], [20, 7], score=True)                  # scores stay as they were


@pytest.mark.parametrize("heads,lens,news", [((4, 1), [9000], [5]), ((8, 2), [7000, 20], [40, 20]), ((8, 8), [4100], [130])], ids=str)
def test_attend_over_a_long_cache(heads, lens, news):
    attend_case(128, heads[0], heads[1], 64, lens, news)


def test_attend_of_many_sequences():
    lens = [1 + (i * 37) % 90 for i in range(700)]
    attend_case(64, 2, 1, 16, lens, [min(n, (i * 7) % 4) for i, n in enumerate(lens)])


@pytest.mark.parametrize("scale", [1e-30, 1e30, 8e36])
def test_attend_with_values_of_any_size(scale):
    attend_case(128, 4, 2, 16, [400, 41], [90, 2], scale=scale, qscale=1.0 / scale)


@pytest.mark.parametrize("page", [4, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_beside_nan(d, page):
    """NaN and infinite powers of two behind the end and where a window hides them reach nobody; NaN of seen entries just the tokens that see them."""
    attend_case(d, 4, 2, page, [70, 33, 16], [20, 33, 1], spoil=lambda t, lens: spoil_hidden(t, torch.tensor(lens)))

    def some(t, lens):
        spoil_hidden(t, torch.tensor(lens))
        for b, at in ((0, 60), (0, 35), (1, 20)):
            p = int(t["table"][b, at // page])
            t["v_exp"][p, b, at % page, d // 64] = -128
        p = int(t["table"][2, 15 // page])
        t["k_exp"][p, 0, 15 % page, 0] = -128
    attend_case(d, 4, 2, page, [70, 33, 16], [20, 33, 5], spoil=some)
    attend_case(d, 4, 2, page, [70, 33, 16], [20, 33, 5], window=12, n_sink=2, spoil=some)

    def late(t, lens):
        spoil_hidden(t, torch.tensor(lens))
        for b, at in ((0, 160), (0, 299), (1, 120)):
            p = int(t["table"][b, at // page])
            t["v_exp"][p, b, at % page, d // 64] = -128
    attend_case(d, 4, 2, page, [300, 233], [170, 133], spoil=late)


def test_attend_with_entries_that_have_no_page():
    def spoil(t, lens):
        t["table"][0, 1], t["table"][1, 0] = -1, t["k"].shape[0] + 3
        t["v_exp"][0] = -128
        t["k_exp"][0] = -128
    for page in (4, 16, 64):
        attend_case(128, 4, 2, page, [3 * page + 1, 2 * page], [page, 3], spoil=spoil)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("total", [14, 18, 22, 30, 60, 100])
def test_logits_of_any_size(d, total):
    """Logits that are products of a power of two and a code, exact in fp32: tokens attend to the highest entry they see, or to those that
    share its value, alone.  Heads in turn: of such logits, of their negatives, of all-zero ones and of small ones."""
    n, m, page = 700, 90, 64
    g = torch.Generator().manual_seed(total)
    code = torch.randint(0, 8, (n,), generator=g)
    k = torch.zeros((n, 2, d))
    k[:, :, 0] = ref.GRID[code].float()[:, None]
    k[:, :, 32] = 6.0 * torch.where(torch.rand(n, generator=g) < 0.5, 1.0, -1.0)[:, None]
    k[:, :, 1] = 6.0  # (every block's power of two is one)
    v = ref.rounded4(torch.randn((n, 2, d), generator=g).to(BF16)).to(BF16)
    t = ref.make_pages4(1, 2, d, page, -(-n // page), 1, score=False, pos=False)
    p, r = pages_ref.entries(t, 0, n)
    for x, y in (("k", k), ("v", v)):
        t[x][p, :, r], t[x + "_exp"][p, :, r] = ref.encode4(y)
    q = torch.zeros((m, 8, d))
    for h, f in enumerate((2.0 ** total, -2.0 ** total, 0.0, 0.25, 2.0 ** total, -2.0 ** total, 0.0, 0.25)):
        q[:, h, 0] = f
        q[:, h, 32] = f / 2 ** 7 if h % 4 == 3 else 0.0
    q = q.to(BF16)
    out = torch.zeros((m, 8, d), dtype=BF16)
    want, tol = ref.attend_ref(ref.values(t), q, [0, m], [n], None, 0, 0, 1 << 20, out)
    # ties and gaps are exact, so the bound's share of the logits' magnitude does not apply to the large ones: their weights are equal or zero
    exact = tol.clone()
    for h in (0, 1, 2, 4, 5, 6):
        exact[:, h] = (2.0 ** -8 * want.abs() + (2.0 ** -15 + n * 2.0 ** -23) * 6.0)[:, h]
    gt = on_gpu(t)
    pages = pages_of(gt, 8)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    og = out.cuda()
    pages.d2o_pages_attend(q.cuda(), i32([0, m]), i32([n]), og)
    within(og, want, exact)
    one = torch.zeros((1, 8, d), dtype=BF16, device="cuda:0")
    pages.d2o_pages_attend(q[-1:].cuda(), i32([0, 1]), i32([n]), one)
    within(one, want[-1:], exact[-1:])
    pages.d2o_pages_step(q[-1:].cuda(), None, None, i32([n]), one)
    within(one, want[-1:], exact[-1:])


def test_large_logits_beside_large_values():
    """Means of values near the largest number where all logits are equal, and large: no sum overflows."""
    n, m, d, page = 5000, 20, 128, 64
    t = ref.make_pages4(1, 1, d, page, -(-n // page), 1, score=False, pos=False)
    t["k"].fill_(0x22), t["k_exp"].zero_()              # all ones
    t["v"].fill_(0x77), t["v_exp"].fill_(125)           # 6 * 2^125
    gt = on_gpu(t)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    for size in (0.0, 2.0 ** 10, 2.0 ** 22, -2.0 ** 40, 2.0 ** 100, -2.0 ** 126):
        q = torch.full((m, 1, d), size / d, dtype=BF16, device="cuda:0")
        out = torch.zeros_like(q)
        pages_of(gt, 1).d2o_pages_attend(q, i32([0, m]), i32([n]), out)
        assert bool((out.float() == 6.0 * 2.0 ** 125).all()), size
        one = torch.zeros((1, 1, d), dtype=BF16, device="cuda:0")
        pages_of(gt, 1).d2o_pages_step(q[:1], None, None, i32([n]), one)
        assert bool((one.float() == 6.0 * 2.0 ** 125).all()), size


def placed(t, how):
    """The same tables at odd places: exponents from an address that is a multiple of 4 alone, or rows further apart than 2^21 bytes."""
    out = on_gpu(t)
    if how == "exponents":
        for x in ("k_exp", "v_exp"):
            room = torch.full((t[x].numel() + 16,), 99, dtype=torch.int8, device="cuda:0")
            out[x] = room[4:4 + t[x].numel()].view(t[x].shape).copy_(t[x])
            assert out[x].data_ptr() % 16 == 4
        return out
    pages, heads, page, wide = t["k"].shape
    for x in ("k", "v"):
        step = (1 << 21) + 64
        room = torch.zeros(pages * page * step, dtype=torch.uint8, device="cuda:0")
        out[x] = torch.as_strided(room, t[x].shape, (page * step, wide, step, 1))
        out[x].copy_(t[x])
    return out


@pytest.mark.parametrize("how", ["exponents", "rows"])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64), (128, 16)])
def test_odd_addresses_and_wide_strides(d, page, how):
    lens, news = [3 * page + 5, page], [page + 3, 1]
    t = ref.make_pages4(2, 2, d, page, 4, 5, score=True, pos=False, spare=0)
    g = torch.Generator().manual_seed(2)
    q = torch.randn((sum(news), 4, d), generator=g).to(BF16)
    first = [0, news[0], sum(news)]
    out = torch.zeros(q.shape, dtype=BF16)
    want, tol = ref.attend_ref(ref.values(t), q, first, lens, None, 0, 0, 4 * page, out)
    gt = placed(t, how)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda:0")  # noqa: E731
    pages, og = pages_of(gt, 4), out.cuda()
    pages.d2o_pages_attend(q.cuda(), i32(first), i32(lens), og)
    within(og, want, tol)
    bits_same(gt, t)
    # a step that stores its tokens, and rows put and read back
    kn, vn = (torch.randn((2, 2, d), generator=g).to(BF16) for _ in range(2))
    n = torch.tensor([x + 1 for x in lens], dtype=torch.int32)
    want, tol, new, add, add_tol = ref.step_ref4(t, q[:2], kn, vn, n, None, 0, 0, 4 * page)
    o = torch.zeros((2, 4, d), dtype=BF16, device="cuda:0")
    pages.d2o_pages_step(q[:2].cuda(), kn.cuda(), vn.cuda(), n.cuda(), o)
    within(o, want, tol)
    same_values(gt, new)
    slots = torch.tensor([5, page + 1, -1], device="cuda:0")
    K, V = (torch.randn((3, 2, d), generator=g).to(BF16).cuda() for _ in range(2))
    pages.d2o_pages_put(K, V, slots)
    Ko, Vo = torch.zeros_like(K), torch.zeros_like(V)
    pages.d2o_pages_get(slots, Ko, Vo)
    assert torch.equal(Ko[:2].cpu().double(), ref.rounded4(K[:2].cpu())) and torch.equal(Vo[:2].cpu().double(), ref.rounded4(V[:2].cpu()))
