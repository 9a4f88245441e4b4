"""Caches in pages - prompts into them, generation steps, evictions - against their 64-bit forms."""
import math

import numpy as np
import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TENSORS = ("k", "v", "k_exp", "v_exp", "score", "pos")


def on_gpu(t):
    out = {}
    for name, x in t.items():
        if x is None:
            out[name] = None
            continue
        y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device="cuda:0")
        y.copy_(x)
        out[name] = y
    return out


def pages_of(t, q_heads, max_len=None):
    return binding.Pages(t["k"], t["v"], t["table"], q_heads, K_exp=t["k_exp"], V_exp=t["v_exp"], score=t["score"],
                         pos=t["pos"], max_len=max_len)


def same(got, want, names=TENSORS):
    for x in names:
        if want[x] is not None:
            g, w = got[x].cpu(), want[x]
            if w.dtype in (F32, BF16):
                g, w = g.view(torch.int32 if w.dtype == F32 else torch.int16), w.view(torch.int32 if w.dtype == F32 else torch.int16)
            assert torch.equal(g, w), x


def cuda(*xs):
    return [None if x is None else x.cuda() for x in xs]


# ---- generation steps ----------------------------------------------------------------------

def step_case(dtype, d, B, Hq, Hkv, page, lens, window=0, n_sink=0, fp8=False, score=True, pos=False, append=True,
              order="pool", seed=0, max_len=None, spoil=None, qscale=1.5, positions=None):
    lens = torch.tensor(lens, dtype=torch.int32)
    cap = -(-max(1, int(lens.max())) // page) + 1
    t = ref.make_pages(B, Hkv, d, page, cap, dtype, seed, fp8, order, score, pos)
    g = torch.Generator().manual_seed(77 + seed)
    q = (torch.randn((B, Hq, d), generator=g) * qscale).to(dtype)
    kn, vn = (torch.randn((B, Hkv, d), generator=g).to(dtype) if append else None for _ in range(2))
    if pos:  # entries in any order, with gaps
        for b in range(B):
            n = int(lens[b])
            p, r = ref.entries(t, b, n)
            for h in range(Hkv):
                t["pos"][p, h, r] = (3 * torch.randperm(n, generator=g)).to(torch.int32) if n else t["pos"][p, h, r]
        if positions is None:
            positions = torch.tensor([3 * max(0, int(n) - 1) + 2 for n in lens], dtype=torch.int32)
    if spoil:
        spoil(t, lens)
    m = max_len or cap * page
    want, tol, new, add, add_tol = ref.step_ref(t, q, kn, vn, lens, positions, window, n_sink, m, dtype)
    gt = on_gpu(t)
    pages = pages_of(gt, Hq, m)
    out = torch.full((B, Hq, d), 7.0, dtype=dtype, device="cuda:0")
    pages.d2o_pages_step(*cuda(q, kn, vn, lens), out, positions=None if positions is None else positions.cuda(), window=window,
                         n_sink=n_sink)
    torch.cuda.synchronize()
    got = out.cpu().double()
    assert bool(torch.isfinite(got).all())
    err = (got - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    same(gt, new, ("k", "v", "k_exp", "v_exp", "pos"))
    if score:
        g64 = gt["score"].cpu().double()
        w64 = new["score"].double() + add
        untouched = add_tol == 0
        assert torch.equal(gt["score"].cpu()[untouched], new["score"][untouched])
        e = (g64 - w64).abs()[~untouched]
        assert bool((e <= add_tol[~untouched]).all()), float((e / add_tol[~untouched]).max())
    return gt


FORMS = [(F32, False), (BF16, False), (BF16, True)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
@pytest.mark.parametrize("heads,page,lens", [
    ((1, 1), 16, [1]), ((2, 1), 1, [2, 1]), ((4, 4), 8, [15, 16, 17]), ((3, 1), 16, [31, 33]), ((8, 1), 64, [63, 64, 65]),
    ((16, 1), 32, [100]), ((10, 2), 128, [127, 129]), ((4, 1), 256, [255, 257, 1]), ((6, 2), 2, [511, 7]),
    ((8, 8), 1024, [1025, 3]), ((2, 2), 64, [2050]), ((4, 2), 16, [700, 0, 5, 1300]), ((11, 1), 4, [77]),
], ids=str)
def test_step(dtype, fp8, d, heads, page, lens):
    step_case(dtype, d, len(lens), heads[0], heads[1], page, lens, fp8=fp8, seed=sum(lens))


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
@pytest.mark.parametrize("window,n_sink,lens", [
    (1, 0, [1, 200]), (16, 4, [500, 17]), (100, 0, [100, 101]), (64, 130, [400, 60]), (1000, 1, [1500, 90]), (3, 3, [6, 7]),
], ids=str)
def test_step_through_a_window(dtype, fp8, pos, window, n_sink, lens):
    step_case(dtype, 128, len(lens), 4, 2, 16, lens, window, n_sink, fp8, pos=pos, seed=window)


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_without_a_new_token_and_without_scores(dtype, fp8):
    step_case(dtype, 128, 2, 8, 2, 32, [300, 41], fp8=fp8, append=False, score=False)
    step_case(dtype, 64, 2, 8, 2, 32, [300, 41], fp8=fp8, append=False, score=True)
    step_case(dtype, 64, 2, 8, 2, 32, [300, 41], fp8=fp8, append=True, score=False)


@pytest.mark.parametrize("heads,n", [((4, 1), 20011), ((32, 8), 9001), ((8, 8), 12288), ((16, 1), 16385)], ids=str)
def test_step_over_a_long_cache(heads, n):
    step_case(BF16, 128, 1, heads[0], heads[1], 64, [n], seed=n)


def test_step_of_many_short_sequences():
    lens = [1 + (i * 37) % 90 for i in range(70)]
    step_case(BF16, 64, len(lens), 4, 2, 16, lens)


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_with_pages_whose_rows_lie_by_token(dtype, fp8):
    step_case(dtype, 128, 2, 4, 2, 16, [100, 37], fp8=fp8, order="token")


@pytest.mark.parametrize("total", [14, 30, 100])
@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_with_logits_of_any_size(dtype, fp8, total):
    """Logits of up to 15 times 2^total, exact in fp32 and steps of 2^total / sqrt(d) apart: a head attends to its highest entry, or to
    those that share its value, alone.  Heads in turn: of such logits, of their negatives, of all-zero ones and of small ones."""
    d, n, Hkv, G = 128, 700, 2, 4
    t = ref.make_pages(1, Hkv, d, 16, n // 16 + 1, dtype, total, fp8)
    t["pos"] = None
    g = torch.Generator().manual_seed(total)
    K = torch.zeros(t["k"].shape)
    K[..., 0] = torch.randint(1, 16, K.shape[:3], generator=g).float() * 2.0 ** (total // 2)
    if fp8:
        t["k"], t["k_exp"] = ref.encode(K.to(BF16))
    else:
        t["k"] = K.to(dtype)
    q = torch.zeros(1, Hkv * G, d)
    q[0, :, 0] = torch.tensor([2.0 ** (total - total // 2), -2.0 ** (total - total // 2), 0.0, 2.0 ** -(total // 2)]).repeat(Hkv)
    q = q.to(dtype)
    lens = torch.tensor([n], dtype=torch.int32)
    gt = on_gpu(t)
    out = torch.empty_like(q, device="cuda:0")
    pages_of(gt, Hkv * G).d2o_pages_step(q.cuda(), None, None, lens.cuda(), out)
    p, r = ref.entries(t, 0, n)
    # the small heads' logits, at most 2, rounded three times, all of them scaled and their exponentials rounded: in the sum and in the normaliser
    rel = 2 * (2 * 3 * 2.0 ** -24 + 2.0 ** -22 + n * 2.0 ** -24)
    for h in range(Hkv):
        k, v = (ref.rows64(t[x], t[x + "_exp"], p, h, r) for x in ("k", "v"))
        o, pr = ref.attend64(q[0, h * G:(h + 1) * G].double(), k, v, torch.ones((G, n), dtype=torch.bool))
        err = (out[0, h * G:(h + 1) * G].cpu().double() - o).abs()
        tol = pr @ v.abs() * rel + o.abs() * ref.HALF_STEP[dtype]
        assert bool((err <= tol).all()), (h, float((err / tol).max()))
        old, now = t["score"][p, h, r].double(), gt["score"].cpu()[p, h, r].double()
        tol = pr.sum(0) * rel + (G + 1) * 2.0 ** -24 * (pr.sum(0) + old) + 1e-38
        assert bool(((now - old - pr.sum(0)).abs() <= tol).all())


def spoil_behind(t, lens):
    """What lies behind a sequence's end, and in pages that nobody has, is NaN and infinite."""
    used = torch.zeros(t["k"].shape[0], t["k"].shape[2], dtype=torch.bool)
    for b, n in enumerate(lens):
        p, r = ref.entries(t, b, int(n))
        used[p, r] = True
    for x, bad in (("k", math.nan), ("v", math.inf)):
        keep = t[x].clone()
        t[x][:] = bad
        t[x].copy_(torch.where(used[:, None, :, None], keep, t[x]))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("append", [True, False])
def test_step_never_looks_behind_a_sequence(dtype, append):
    step_case(dtype, 128, 3, 4, 2, 32, [33, 1, 250], spoil=spoil_behind, append=append)
    step_case(dtype, 64, 3, 4, 2, 32, [33, 1, 250], window=20, n_sink=2, spoil=spoil_behind, append=append)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pos", [False, True], ids=["slots", "positions"])
def test_step_masked_rows_that_are_not_finite_take_no_part(dtype, pos):
    def spoil(t, lens):
        for b, n in enumerate(lens):
            p, r = ref.entries(t, b, int(n))
            for h in range(t["k"].shape[1]):
                at = t["pos"][p, h, r] if pos else torch.arange(int(n))
                last = 3 * (int(n) - 1) + 2 if pos else int(n) - 1
                hidden = ~((at > last - 30) | (at < 4))
                t["k"][p[hidden], h, r[hidden]] = math.inf
                t["v"][p[hidden], h, r[hidden]] = math.nan
    step_case(dtype, 128, 2, 4, 2, 16, [200, 75], window=30, n_sink=4, pos=pos, spoil=spoil)


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_pages_that_do_not_exist_are_skipped(dtype, fp8):
    def spoil(t, lens):
        t["table"][0, 1], t["table"][0, 3], t["table"][1, :] = -1, 1 << 30, t["k"].shape[0]
        t["table"][2, int(lens[2] - 1) // 16] = -7  # the new token has no page
    step_case(dtype, 128, 3, 4, 2, 16, [100, 40, 33], fp8=fp8, spoil=spoil)


def test_step_a_window_that_shows_nothing_gives_zeros():
    # positions far behind the new token, which has no page of its own
    def spoil(t, lens):
        t["table"][0, 2] = -1
    step_case(BF16, 128, 1, 4, 2, 16, [33], window=1, spoil=spoil)


def test_step_lengths_beyond_max_len_are_cut_and_store_nothing():
    step_case(BF16, 128, 2, 4, 2, 16, [100, 30], max_len=48)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_step_sharp_attention(dtype):
    step_case(dtype, 128, 1, 4, 2, 16, [600], qscale=60.0)


def test_step_nan_and_infinite_rows_that_are_seen_reach_their_heads_only():
    t = ref.make_pages(1, 2, 128, 16, 8, BF16, 3, score=False, pos=False)
    p, r = ref.entries(t, 0, 100)
    t["v"][p[40], 0, r[40], 5] = math.inf
    t["k"][p[50], 1, r[50], 5] = math.nan
    q = torch.randn((1, 4, 128), generator=torch.Generator().manual_seed(1)).to(BF16)
    gt = on_gpu(t)
    out = torch.zeros((1, 4, 128), dtype=BF16, device="cuda:0")
    pages_of(gt, 4).d2o_pages_step(q.cuda(), None, None, torch.tensor([100], dtype=torch.int32, device="cuda:0"), out)
    got = out.cpu()[0]
    assert bool((got[:2, 5] == math.inf).all()) and bool(torch.isfinite(got[:2, [i for i in range(128) if i != 5]]).all())
    assert bool(got[2:].isnan().all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_step_of_many_heads_per_group_with_rows_and_queries_that_are_not_finite(dtype):
    """An infinite value reaches its column, a NaN key the heads of its group, a NaN query its own head, and nothing else."""
    G, n = 11, 300
    t = ref.make_pages(1, 2, 64, 16, 20, dtype, 3, score=False, pos=False)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((1, 2 * G, 64), generator=g).to(dtype)
    clean = ref.step_ref(t, q, None, None, [n], None, 0, 0, 320, dtype)
    p, r = ref.entries(t, 0, n)
    t["v"][p[40], 0, r[40], 5] = math.inf
    t["k"][p[50], 1, r[50], 5] = math.nan
    q[0, 3] = math.nan
    gt = on_gpu(t)
    out = torch.zeros((1, 2 * G, 64), dtype=dtype, device="cuda:0")
    pages_of(gt, 2 * G).d2o_pages_step(q.cuda(), None, None, torch.tensor([n], dtype=torch.int32, device="cuda:0"), out)
    got = out.cpu()[0].double()
    heads, cols = [h for h in range(G) if h != 3], [c for c in range(64) if c != 5]
    assert bool((got[heads, 5] == math.inf).all()) and bool(got[3].isnan().all()) and bool(got[G:].isnan().all())
    err = (got - clean[0][0]).abs()[heads][:, cols]
    assert bool((err <= clean[1][0][heads][:, cols]).all())


def test_step_strided_queries_and_outputs():
    t = ref.make_pages(2, 2, 64, 16, 8, BF16, 3)
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((2, 9, 80), generator=g).to(BF16).cuda()
    q, kn, vn = wide[:, :4, :64], wide[:, 4:6, :64], wide[:, 6:8, :64]
    lens = torch.tensor([100, 17], dtype=torch.int32, device="cuda:0")
    outs = []
    for a in ((q, kn, vn), (q.contiguous(), kn.contiguous(), vn.contiguous())):
        gt = on_gpu(t)
        out = torch.full((2, 5, 80), 7.0, dtype=BF16, device="cuda:0")
        pages_of(gt, 4).d2o_pages_step(*a, lens, out[:, :4, :64])
        outs.append((out, gt))
    assert torch.equal(outs[0][0], outs[1][0]) and bool((outs[0][0][:, 4:] == 7).all()) and bool((outs[0][0][..., 64:] == 7).all())
    same(outs[0][1], {x: (None if y is None else y.cpu()) for x, y in outs[1][1].items()})


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_repeats_bit_for_bit(dtype, fp8):
    """The order of every sum is fixed, whatever the workgroups' order: five runs on equal pages agree, on two streams."""
    t = ref.make_pages(3, 2, 128, 32, 100, dtype, 9, fp8)
    g = torch.Generator().manual_seed(2)
    q, kn, vn = ((torch.randn((3, h, 128), generator=g)).to(dtype).cuda() for h in (8, 2, 2))
    lens = torch.tensor([3200, 700, 1], dtype=torch.int32, device="cuda:0")
    first = None
    side = torch.cuda.Stream()
    for i in range(5):
        gt = on_gpu(t)
        out = torch.zeros((3, 8, 128), dtype=dtype, device="cuda:0")
        torch.cuda.synchronize()
        with torch.cuda.stream(side if i % 2 else torch.cuda.current_stream()):
            pages_of(gt, 8).d2o_pages_step(q, kn, vn, lens, out)
        torch.cuda.synchronize()
        got = {**{x: (None if y is None else y.cpu()) for x, y in gt.items()}, "out": out.cpu()}
        first = first or got
        same(got, first)
        assert torch.equal(got["out"], first["out"])


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_step_over_pages_that_sequences_share(dtype, fp8):
    """Three sequences with one prompt's pages in front and a page each of their own, where the new rows go; no scores are kept."""
    t = ref.make_pages(3, 2, 64, 16, 8, dtype, 12, fp8, score=False, pos=False)
    t["table"][1:, :6] = t["table"][0, :6]
    g = torch.Generator().manual_seed(12)
    q, kn, vn = (torch.randn((3, h, 64), generator=g).to(dtype) for h in (6, 2, 2))
    lens = torch.tensor([100, 97, 112], dtype=torch.int32)
    want, tol, new, _, _ = ref.step_ref(t, q, kn, vn, lens, None, 0, 0, 128, dtype)
    gt = on_gpu(t)
    out = torch.zeros((3, 6, 64), dtype=dtype, device="cuda:0")
    pages_of(gt, 6).d2o_pages_step(*cuda(q, kn, vn, lens), out)
    assert bool(((out.cpu().double() - want).abs() <= tol).all())
    same(gt, new)


@pytest.mark.parametrize("positions", [[5, 0], [199, 35], [260, 45], [0x7FFFFFFF, 41]], ids=str)
def test_step_positions_that_are_not_the_entry(positions):
    """Pages without positions: entry s has position s, and the window ends at the position that is given."""
    step_case(BF16, 64, 2, 4, 2, 16, [200, 40], window=70, n_sink=3, positions=torch.tensor(positions, dtype=torch.int32))


def test_step_exponents_at_odd_addresses():
    t = ref.make_pages(2, 2, 128, 32, 8, BF16, 5, fp8=True)
    g = torch.Generator().manual_seed(5)
    q, kn, vn = (torch.randn((2, h, 128), generator=g).to(BF16).cuda() for h in (8, 2, 2))
    lens = torch.tensor([230, 33], dtype=torch.int32, device="cuda:0")
    got = []
    for shift in (0, 1, 3):
        gt = on_gpu(t)
        for x in ("k_exp", "v_exp"):
            flat = torch.empty(t[x].numel() + shift, dtype=torch.int8, device="cuda:0")[shift:]
            gt[x] = flat.view(t[x].shape)
            gt[x].copy_(t[x])
        out = torch.zeros((2, 8, 128), dtype=BF16, device="cuda:0")
        pages_of(gt, 8).d2o_pages_step(q, kn, vn, lens, out)
        got.append((out, {x: (None if y is None else y.cpu()) for x, y in gt.items()}))
    for out, tensors in got[1:]:
        assert torch.equal(out, got[0][0])
        same(tensors, got[0][1])


def test_two_caches_at_once_on_two_streams():
    """An object each, the same pages read by both: neither disturbs the other."""
    t = ref.make_pages(4, 4, 128, 64, 64, BF16, 14, score=False, pos=False)
    gt = on_gpu(t)
    g = torch.Generator().manual_seed(14)
    qs = [torch.randn((4, 16, 128), generator=g).to(BF16).cuda() for _ in range(2)]
    lens = [torch.tensor(x, dtype=torch.int32, device="cuda:0") for x in ([4096, 4000, 77, 1], [900, 4096, 4096, 4095])]
    pages, outs, want = [pages_of(gt, 16) for _ in range(2)], [], []
    for p, q, n in zip(pages, qs, lens):
        want.append(torch.zeros_like(q))
        p.d2o_pages_step(q, None, None, n, want[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i in range(20):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                outs.append(torch.zeros_like(qs[j]))
                pages[j].d2o_pages_step(qs[j], None, None, lens[j], outs[-1])
    torch.cuda.synchronize()
    assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))


def test_fill_and_evictions_captured_and_replayed():
    """A graph of a prompt in slices, a shorter one and evictions with moves in a launch of their own and without, replayed with new inputs."""
    n, B, Hkv, d = 20000, 2, 2, 64
    t = ref.make_pages(B, Hkv, d, 64, 41, BF16, 15)
    a, b = on_gpu(t), on_gpu(t)
    pa, pb = pages_of(a, Hkv, n), pages_of(b, Hkv, n)
    K, V = (torch.zeros((B, Hkv, n, d), dtype=BF16, device="cuda:0") for _ in range(2))
    sc = torch.zeros((B, Hkv, n), device="cuda:0")
    lens, kept = (torch.zeros(B, dtype=torch.int32, device="cuda:0") for _ in range(2))
    half = n // 2

    def work(p):
        p.d2o_pages_fill(K, V, 2600, 300, 4, score=sc, lens=lens)
        p.d2o_pages_evict(kept, 1300, 100, 4)
        p.d2o_pages_fill(K[:, :, :half], V[:, :, :half], 1000, 10, 0, score=sc[:, :, :half].contiguous(), lens=lens)
        p.d2o_pages_evict(kept.clamp(max=1000), 999, 10, 0)

    g = torch.Generator().manual_seed(15)
    work(pa), work(pb)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(pa)
    for m in ([20000, 2700], [12000, 15], [0, 20000], [2601, 19000]):
        K.copy_(torch.randn(K.shape, generator=g)), V.copy_(torch.randn(V.shape, generator=g))
        sc.copy_(torch.rand(sc.shape, generator=g))
        lens.copy_(torch.tensor(m, dtype=torch.int32)), kept.copy_(lens.clamp(max=2600))
        graph.replay()
        torch.cuda.synchronize()
        work(pb)
        torch.cuda.synchronize()
        same(a, {x: (None if y is None else y.cpu()) for x, y in b.items()})


def test_step_captured_and_replayed():
    """A graph of two steps and an eviction sharing a workspace, replayed with new inputs and lengths."""
    t = ref.make_pages(2, 2, 128, 16, 30, BF16, 4)
    g = torch.Generator().manual_seed(3)

    def new(h):
        return torch.randn((2, h, 128), generator=g).to(BF16).cuda()

    a, b = on_gpu(t), on_gpu(t)
    q, kn, vn, out, out2 = new(4), new(2), new(2), new(4), new(4)
    lens = torch.tensor([400, 33], dtype=torch.int32, device="cuda:0")
    pa, pb = pages_of(a, 4), pages_of(b, 4)

    def work(p):
        p.d2o_pages_step(q, kn, vn, lens, out)
        p.d2o_pages_step(q, None, None, lens, out2, window=50, n_sink=2)
        p.d2o_pages_evict(lens, 30, 10, 2)

    work(pa), work(pb)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(pa)
    for i in range(4):
        for x, y in ((q, new(4)), (kn, new(2)), (vn, new(2))):
            x.copy_(y)
        lens.copy_(torch.tensor([100 + 90 * i, 29 + 40 * i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), out2.clone()
        work(pb)
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], out2)
        same(a, {x: (None if y is None else y.cpu()) for x, y in b.items()})


# ---- prompts into pages --------------------------------------------------------------------

def fill_case(dtype, d, B, Hkv, n, lens, budget, recent, n_sink, page, fp8=False, scores=True, order="pool", seed=0,
              spoil=None, keep=True, ties=False):
    per = -(-min(n, budget) // page) + 1
    t = ref.make_pages(B, Hkv, d, page, per, dtype, seed, fp8, order, keep, keep)
    g = torch.Generator().manual_seed(55 + seed)
    K, V = (torch.randn((B, Hkv, n, d), generator=g).to(dtype) for _ in range(2))
    sc = None
    if scores:
        sc = torch.randn((B, Hkv, n), generator=g).exp()
        if ties:
            sc = torch.round(sc)
    if spoil:
        spoil(t, K, V, sc)
    L = [n] * B if lens is None else lens
    want = ref.fill_ref(t, K, V, L, sc, budget, recent, n_sink)
    gt = on_gpu(t)
    pages_of(gt, Hkv, n).d2o_pages_fill(*cuda(K, V), budget, recent, n_sink, score=None if sc is None else sc.cuda(),
                                        lens=None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda:0"))
    torch.cuda.synchronize()
    same(gt, want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
@pytest.mark.parametrize("n,lens,budget,recent,n_sink,page", [
    (1, None, 1, 0, 0, 1), (2, None, 1, 1, 0, 16), (5, [5, 0, 3], 4, 1, 1, 2), (100, None, 100, 0, 0, 16),
    (100, [100, 40, 41], 40, 10, 4, 8), (1000, [1000, 999, 1], 128, 32, 0, 64), (1025, None, 1, 0, 0, 16),
    (1025, None, 1024, 1000, 24, 128), (5000, [5000, 4097], 513, 0, 7, 32), (300, None, 400, 30, 3, 1024), (2049, None, 300, 300, 0, 4),
], ids=str)
def test_fill(dtype, fp8, d, n, lens, budget, recent, n_sink, page):
    fill_case(dtype, d, len(lens) if lens else 2, 3, n, lens, budget, recent, n_sink, page, fp8, seed=n)


@pytest.mark.parametrize("n", [700, 3000, 20000])
def test_fill_with_many_equal_scores(n):
    fill_case(BF16, 64, 2, 2, n, None, n // 5, n // 20, 2, 16, ties=True)
    fill_case(BF16, 64, 1, 2, n, None, n // 5, n // 20, 2, 16, spoil=lambda t, K, V, s: s.zero_())


def test_fill_long_prompt():
    fill_case(BF16, 64, 1, 2, 70001, None, 3501, 800, 4, 64)


def test_fill_long_prompts_of_different_lengths():
    """One batch in which a prompt is long, one short of the budget, one shorter than what a workgroup holds, and one empty."""
    fill_case(BF16, 64, 5, 2, 20001, [20001, 300, 16000, 0, 4097], 500, 100, 3, 16, seed=1)
    fill_case(F32, 64, 2, 1, 20001, [17000, 18000], 500, 497, 3, 16, seed=2)  # nothing but what is protected
    fill_case(BF16, 128, 1, 1, 40000, [36865], 36864, 5, 0, 128, fp8=True, seed=3)


def test_fill_long_prompts_with_scores_that_are_not_finite():
    def spoil(t, K, V, s):
        s[..., 10::50] = math.nan
        s[..., 20::50] = math.inf
        s[..., 30::50] = -math.inf
        s[..., 31::3] = 0.25
    for budget in (300, 1000, 12000):
        fill_case(BF16, 64, 1, 2, 20000, None, budget, 20, 2, 16, spoil=spoil)


def test_fill_scores_that_are_not_finite():
    def spoil(t, K, V, s):
        s[..., 10::50] = math.nan
        s[..., 20::50] = math.inf
        s[..., 30::50] = -math.inf
        s[..., 31::50] = -1.0
        s[..., 32::50] = -0.0
        s[..., 33::50] = 0.0
    fill_case(F32, 64, 1, 2, 600, None, 100, 20, 0, 16, spoil=spoil)
    fill_case(F32, 64, 1, 2, 600, None, 560, 20, 0, 16, spoil=spoil)


def test_fill_without_scores_or_without_keeping_them():
    fill_case(BF16, 128, 2, 2, 50, [50, 20], 60, 0, 0, 16, scores=False)
    fill_case(BF16, 128, 2, 2, 50, [50, 20], 30, 5, 0, 16, keep=False)
    fill_case(BF16, 128, 2, 2, 90, [90, 20], 30, 5, 0, 16, order="token")


def test_fill_skips_pages_that_do_not_exist():
    def spoil(t, K, V, s):
        t["table"][0, 1], t["table"][1, 0], t["table"][1, 2] = -1, t["k"].shape[0], 1 << 30
    fill_case(BF16, 128, 2, 2, 200, None, 64, 10, 0, 16, spoil=spoil)


def test_fill_strided_prompts():
    t = ref.make_pages(2, 2, 64, 16, 4, F32, 8)
    g = torch.Generator().manual_seed(8)
    wide = torch.randn((2, 100, 5, 80), generator=g).cuda()
    K, V = wide[:, :, :2, :64].transpose(1, 2), wide[:, :, 2:4, :64].transpose(1, 2)
    sc = torch.rand((2, 2, 100), generator=g)
    want = ref.fill_ref(t, K.cpu(), V.cpu(), [100, 100], sc, 40, 10, 0)
    gt = on_gpu(t)
    pages_of(gt, 2, 100).d2o_pages_fill(K, V, 40, 10, 0, score=sc.cuda())
    same(gt, want)


# ---- evictions -----------------------------------------------------------------------------

def evict_case(dtype, d, B, Hkv, page, lens, budget, recent, n_sink, fp8=False, order="pool", seed=0, spoil=None, ties=False,
               max_len=None):
    per = -(-max(lens) // page) + 1
    t = ref.make_pages(B, Hkv, d, page, per, dtype, seed, fp8, order)
    g = torch.Generator().manual_seed(66 + seed)
    for b, n in enumerate(lens):
        p, r = ref.entries(t, b, n)
        for h in range(Hkv):
            t["pos"][p, h, r] = (2 * torch.randperm(n, generator=g)).to(torch.int32)
            if ties:
                t["score"][p, h, r] = torch.round(4 * t["score"][p, h, r])
    if spoil:
        spoil(t, lens)
    want = ref.evict_ref(t, lens, budget, recent, n_sink)
    gt = on_gpu(t)
    pages_of(gt, Hkv, max_len).d2o_pages_evict(torch.tensor(lens, dtype=torch.int32, device="cuda:0"), budget, recent, n_sink)
    torch.cuda.synchronize()
    same(gt, want)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
@pytest.mark.parametrize("lens,budget,recent,n_sink,page", [
    ([2], 1, 0, 0, 1), ([2, 1, 0], 1, 1, 0, 16), ([17, 16, 18], 16, 4, 2, 4), ([129, 128], 128, 32, 4, 16), ([1025], 1024, 1000, 0, 64),
    ([1500, 1600], 1, 0, 0, 32), ([300], 299, 299, 0, 8), ([2304, 2100], 2048, 2000, 4, 64), ([4000], 100, 10, 50, 1024),
    ([5000, 3], 4000, 0, 0, 128), ([1639, 1639], 1638, 409, 0, 64),
], ids=str)
def test_evict(dtype, fp8, d, lens, budget, recent, n_sink, page):
    evict_case(dtype, d, len(lens), 2, page, lens, budget, recent, n_sink, fp8, seed=sum(lens))


@pytest.mark.parametrize("over", [1, 2, 65, 300])
def test_evict_equal_scores(over):
    evict_case(BF16, 64, 2, 2, 16, [400 + over, 350], 400, 30, 3, ties=True)
    evict_case(BF16, 64, 1, 2, 16, [400 + over], 400, 0, 0, spoil=lambda t, lens: t["score"].zero_())


@pytest.mark.parametrize("over", [1, 40])
def test_evict_the_same_position_twice(over):
    """Entries with equal score and position: the lower entry is kept, and exactly `budget` entries are."""
    def spoil(t, lens):
        t["pos"].fill_(5)
        t["score"].fill_(1.0)
    evict_case(BF16, 64, 1, 2, 16, [200 + over], 200, 10, 3, spoil=spoil)
    evict_case(BF16, 64, 1, 2, 16, [200 + over], 200, 10, 30, spoil=spoil)

    def twins(t, lens):
        p, r = ref.entries(t, 0, lens[0])
        t["pos"][p[1::2], :, r[1::2]] = t["pos"][p[0:-1:2], :, r[0:-1:2]][:len(p[1::2])]
        t["score"][p, :, r] = torch.round(3 * t["score"][p, :, r])
    evict_case(BF16, 64, 1, 2, 16, [200 + over], 200, 10, 30, spoil=twins)


@pytest.mark.parametrize("n_sink,recent", [(300, 0), (0, 200), (3, 10)])
@pytest.mark.parametrize("lens,budget", [([201], 200), ([240], 200), ([5000], 4999), ([5000], 4000), ([17001], 17000), ([17001], 300)],
                         ids=str)
def test_evict_more_protected_entries_than_stay(lens, budget, n_sink, recent):
    """Positions that occur many times, all protected: then the scores decide among them too."""
    def spoil(t, lens):
        p, r = ref.entries(t, 0, lens[0])
        t["pos"][p, :, r] = torch.where(torch.arange(lens[0])[:, None] % 50 == 7, 1000, 5 if n_sink > 5 else 2000).to(torch.int32).expand(-1, 2)
        t["score"][p[::3], :, r[::3]] = 0.5
    evict_case(BF16, 64, 1, 2, 16, lens, budget, min(recent, budget - min(n_sink, budget)), min(n_sink, budget), spoil=spoil)


def test_evict_again_what_was_not_shortened():
    """A second call on the same lengths meets entries that were moved and still lie behind the budget: each position twice."""
    t = ref.make_pages(1, 2, 64, 16, 30, BF16, 12)
    g = torch.Generator().manual_seed(12)
    p, r = ref.entries(t, 0, 400)
    for h in range(2):
        t["pos"][p, h, r] = torch.cat([torch.randperm(300, generator=g), torch.arange(300, 400)]).to(torch.int32)
    gt = on_gpu(t)
    pages = pages_of(gt, 2)
    lens = torch.tensor([400], dtype=torch.int32, device="cuda:0")
    for _ in range(3):
        t = ref.evict_ref(t, [400], 300, 250, 4)
        pages.d2o_pages_evict(lens, 300, 250, 4)
        same(gt, t)


@pytest.mark.parametrize("over", [1, 50])
def test_evict_scores_that_are_not_finite_and_any_positions(over):
    def spoil(t, lens):
        for b, n in enumerate(lens):
            p, r = ref.entries(t, b, n)
            t["score"][p[::7], :, r[::7]] = math.nan
            t["score"][p[1::7], :, r[1::7]] = math.inf
            t["score"][p[2::7], :, r[2::7]] = -math.inf
            t["score"][p[3::7], :, r[3::7]] = -0.0
            t["score"][p[4::7], :, r[4::7]] = 0.0
            t["pos"][p[5::7], :, r[5::7]] = -3
            t["pos"][p[6::21], :, r[6::21]] = 0x7FFFFFFF
    evict_case(F32, 64, 2, 2, 16, [300 + over, 310 + over], 300, 20, 2, spoil=spoil)


@pytest.mark.parametrize("over", [1, 30])
def test_evict_with_pages_that_do_not_exist(over):
    def spoil(t, lens):
        t["table"][0, 1], t["table"][0, (lens[0] - 1) // 16], t["table"][1, :] = -1, 1 << 30, -1
    evict_case(BF16, 64, 2, 2, 16, [100 + over, 100 + over], 100, 20, 2, spoil=spoil)


@pytest.mark.parametrize("lens,budget", [([40001], 40000), ([30000], 3000), ([20300], 20000), ([50000], 30000)], ids=str)
def test_evict_long_caches(lens, budget):
    evict_case(BF16, 64, 1, 1, 64, lens, budget, budget // 4, 4)


def _equal(t, lens):
    t["score"].fill_(0.25)


def _one_position(t, lens):
    t["score"].fill_(0.25)
    t["pos"].fill_(9)


def _not_finite(t, lens):
    for i, x in enumerate((math.nan, math.inf, -math.inf, -0.0, 0.0)):
        for b, n in enumerate(lens):
            p, r = ref.entries(t, b, n)
            t["score"][p[i::9], :, r[i::9]] = x
            t["pos"][p[5::18], :, r[5::18]] = -3


def _protected(t, lens):
    """Nearly all entries have the newest position."""
    for b, n in enumerate(lens):
        p, r = ref.entries(t, b, n)
        t["pos"][p[10:], :, r[10:]] = 1 << 20
        t["score"][p[::3], :, r[::3]] = 0.5


def _no_pages(t, lens):
    for b, n in enumerate(lens):
        t["table"][b, 1 + b], t["table"][b, (n - 1) // 64], t["table"][b, 100] = -1, 1 << 30, -5


def _ascending(t, lens):
    """Everything that goes lies in one slice."""
    for b, n in enumerate(lens):
        p, r = ref.entries(t, b, n)
        t["score"][p, :, r] = (torch.arange(n) if b == 0 else n - torch.arange(n)).float()[:, None].expand(-1, t["score"].shape[1])


@pytest.mark.parametrize("spoil", [None, _equal, _one_position, _not_finite, _protected, _no_pages, _ascending],
                         ids=lambda f: f.__name__[1:] if f else "plain")
@pytest.mark.parametrize("budget,over", [(16384, 1), (17000, 37), (20470, 512), (33000, 513), (16390, 200)], ids=str)
def test_evict_a_few_of_long_caches(budget, over, spoil):
    """Sequences that give up as many as there may be, half of them, one and none."""
    evict_case(BF16, 64, 4, 1, 64, [budget + over, budget + max(1, over // 2), budget + 1, budget], budget, 300, 4, spoil=spoil, ties=over == 37,
               max_len=budget + over, seed=over)


@pytest.mark.parametrize("dtype,fp8", FORMS, ids=["f32", "bf16", "fp8"])
def test_evict_one_of_a_long_cache_of_many_heads(dtype, fp8):
    evict_case(dtype, 128, 1, 5, 16, [70001], 70000, 17500, 4, fp8, max_len=70016)


def test_evict_rows_by_token_and_lengths_beyond_max_len():
    evict_case(BF16, 128, 2, 2, 16, [100, 130], 90, 20, 2, order="token")
    # a sequence that claims more than max_len is cut to it
    t = ref.make_pages(1, 2, 64, 16, 10, F32, 1)
    want = ref.evict_ref(t, [64], 50, 5, 0)
    gt = on_gpu(t)
    pages_of(gt, 2, 64).d2o_pages_evict(torch.tensor([150], dtype=torch.int32, device="cuda:0"), 50, 5, 0)
    same(gt, want)


@pytest.mark.parametrize("page", [16, 4])
def test_pools_beyond_32_bits(page):
    """A pool of 9 GiB of which a few pages at its end are in use: prompts, a step and an eviction."""
    Hkv, d, per = 2, 128, -(-80 // page)
    n_pages = (9 << 30) // (2 * page * Hkv * d)
    t = ref.make_pages(1, Hkv, d, page, per, BF16, 21, spare=0)
    g = torch.Generator().manual_seed(21)
    K, V = (torch.randn((1, Hkv, 100, d), generator=g).to(BF16) for _ in range(2))
    sc = torch.rand((1, Hkv, 100), generator=g)
    q, kn, vn = (torch.randn((1, h, d), generator=g).to(BF16) for h in (4, 2, 2))
    lens = torch.tensor([71], dtype=torch.int32)
    at = torch.tensor([100], dtype=torch.int32)
    big = {}
    for x in ("k", "v", "score", "pos"):
        big[x] = torch.empty((n_pages,) + t[x].shape[1:], dtype=t[x].dtype, device="cuda:0")
        big[x][n_pages - per:] = t[x].cuda()
    table = (t["table"] + (n_pages - per)).cuda()
    p = binding.Pages(big["k"], big["v"], table, 4, score=big["score"], pos=big["pos"], max_len=100)
    p.d2o_pages_fill(*cuda(K, V), 70, 20, 2, score=sc.cuda())
    t = ref.fill_ref(t, K, V, [100], sc, 70, 20, 2)
    want, tol, t, add, add_tol = ref.step_ref(t, q, kn, vn, lens, at, 0, 0, 80, BF16)
    out = torch.zeros((1, 4, d), dtype=BF16, device="cuda:0")
    p.d2o_pages_step(*cuda(q, kn, vn, lens), out, positions=at.cuda())
    assert bool(((out.cpu().double() - want).abs() <= tol).all())
    t["score"] = big["score"][n_pages - per:].cpu()
    p.d2o_pages_evict(lens.cuda(), 60, 20, 2)
    t = ref.evict_ref(t, [71], 60, 20, 2)
    same({x: (None if t[x] is None else big[x][n_pages - per:]) for x in TENSORS}, t)


# ---- as they are used together --------------------------------------------------------------

def test_wrong_arguments_are_refused():
    t = on_gpu(ref.make_pages(2, 2, 64, 16, 4, BF16, 0))
    p = pages_of(t, 4)
    lens = torch.tensor([3, 4], dtype=torch.int32, device="cuda:0")
    q, kn = torch.zeros((2, 4, 64), dtype=BF16, device="cuda:0"), torch.zeros((2, 2, 64), dtype=BF16, device="cuda:0")
    K = torch.zeros((2, 2, 10, 64), dtype=BF16, device="cuda:0")
    bare = binding.Pages(t["k"], t["v"], t["table"], 4)
    bad = [
        lambda: binding.Pages(t["k"], t["v"], t["table"], 5),
        lambda: binding.Pages(t["k"], t["v"], t["table"], 34),
        lambda: binding.Pages(t["k"], t["v"][:, :1], t["table"], 4),
        lambda: binding.Pages(t["k"].cpu(), t["v"], t["table"], 4),
        lambda: binding.Pages(t["k"], t["v"], t["table"].long(), 4),
        lambda: binding.Pages(t["k"], t["v"], t["table"], 4, K_exp=t["score"], V_exp=t["score"]),
        lambda: binding.Pages(t["k"], t["v"], t["table"], 4, score=t["pos"]),
        lambda: binding.Pages(t["k"][:, :, :12], t["v"][:, :, :12], t["table"], 4),
        lambda: binding.Pages(t["k"].view(torch.uint8), t["v"].view(torch.uint8), t["table"], 4),
        lambda: binding.Pages(t["k"], t["v"], t["table"], 4, max_len=0),
        lambda: p.d2o_pages_step(q, kn, None, lens, q),
        lambda: p.d2o_pages_step(q.float(), kn, kn, lens, q),
        lambda: p.d2o_pages_step(q, kn, kn, lens[:1], q),
        lambda: p.d2o_pages_step(q, kn, kn, lens.long(), q),
        lambda: p.d2o_pages_step(q, kn, kn, lens, q, window=-1),
        lambda: p.d2o_pages_step(q, kn, kn, lens, q, n_sink=-1),
        lambda: p.d2o_pages_step(q, kn, kn, lens, q, positions=lens.cpu()),
        lambda: p.d2o_pages_fill(K, K, 0),
        lambda: p.d2o_pages_fill(K, K, 9, score=None),
        lambda: p.d2o_pages_fill(K, K[:, :, :9], 20),
        lambda: p.d2o_pages_fill(K, K, 9, 5, 5, score=torch.zeros((2, 2, 10), device="cuda:0")),
        lambda: p.d2o_pages_fill(torch.zeros((2, 2, 100, 64), dtype=BF16, device="cuda:0"),
                                 torch.zeros((2, 2, 100, 64), dtype=BF16, device="cuda:0"), 100),
        lambda: p.d2o_pages_evict(lens, 0),
        lambda: p.d2o_pages_evict(lens, (1 << 32) + 2),
        lambda: p.d2o_pages_step(q, kn, kn, lens, q, window=1 << 32),
        lambda: p.d2o_pages_evict(lens, 10, 9, 2),
        lambda: bare.d2o_pages_evict(lens, 10),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(binding.D2OError):
            call()
            print("not refused:", i)


def test_window_over_a_prompt_is_a_step_per_token():
    """The prompt form and the single-token form of the same attention: every row of one against a step of the other."""
    Hq, Hkv, n, d, W, T = 4, 2, 90, 64, 25, 3
    g = torch.Generator().manual_seed(4)
    Q, K, V = (torch.randn((1, h, n, d), generator=g).to(F32).cuda() for h in (Hq, Hkv, Hkv))
    want = binding.d2o_window_attend(Q, K, V, W, T)
    t = on_gpu(ref.make_pages(1, Hkv, d, 8, 12, F32, 4, score=False, pos=False))
    p = pages_of(t, Hq)
    out = torch.zeros((1, Hq, d), device="cuda:0")
    for i in range(n):
        p.d2o_pages_step(Q[:, :, i], K[:, :, i], V[:, :, i], torch.tensor([i + 1], dtype=torch.int32, device="cuda:0"), out,
                         window=W, n_sink=T)
        # both are within the bound of the same exact row; rows are means of values below 5
        assert float((out - want[:, :, i]).abs().max()) <= 2 * 5 * (2 * (16 * 67 + 64 + 100) * 2.0 ** -24)


@pytest.mark.parametrize("dtype,fp8", [(BF16, False), (BF16, True), (F32, False)], ids=["bf16", "fp8", "f32"])
def test_prompt_then_generation_with_eviction(dtype, fp8):
    """A prompt through the library's attention with scores, its best tokens into pages, then steps with one eviction each:
    outputs and scores against the 64-bit form at every step, and every eviction the one that the scores in the pages ask for."""
    Hq, Hkv, n, d, S, M, steps, page = 4, 2, 200, 128, 48, 12, 20, 16
    g = torch.Generator().manual_seed(6)
    Q, K, V = (torch.randn((1, h, n, d), generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
    ctx = binding.D2O(1, 1, Hq, Hkv, d, n, S + 8, dtype="f32" if dtype == F32 else "bf16")
    ctx.d2o_prefill_attend(0, *cuda(Q, K, V))
    sc = torch.from_numpy(ctx.d2o_scores_export(0, n))
    ctx.close()
    t = ref.make_pages(1, Hkv, d, page, -(-(S + 1) // page), dtype, 6, fp8)
    gt = on_gpu(t)
    p = pages_of(gt, Hq, n)
    p.d2o_pages_fill(*cuda(K, V), S, M, 2, score=sc.cuda())
    t = ref.fill_ref(t, K, V, [n], sc, S, M, 2)
    same(gt, t)
    lens = torch.tensor([S + 1], dtype=torch.int32)
    lens_d = lens.cuda()
    for i in range(steps):
        q, kn, vn = (torch.randn((1, h, d), generator=g).to(dtype) for h in (Hq, Hkv, Hkv))
        at = torch.tensor([n + i], dtype=torch.int32)
        want, tol, t, add, add_tol = ref.step_ref(t, q, kn, vn, lens, at, 0, 0, S + 1, dtype)
        out = torch.zeros((1, Hq, d), dtype=dtype, device="cuda:0")
        p.d2o_pages_step(*cuda(q, kn, vn), lens_d, out, positions=at.cuda())
        assert bool(((out.cpu().double() - want).abs() <= tol).all())
        got = gt["score"].cpu()
        assert bool(((got.double() - t["score"].double() - add).abs() <= add_tol).all())
        t["score"] = got  # (fp32 sums: the library's own decide the eviction)
        p.d2o_pages_evict(lens_d, S, M, 2)
        t = ref.evict_ref(t, [S + 1], S, M, 2)
        same(gt, t)
    kept = gt["pos"].cpu()[t["table"][0].long()].transpose(0, 1).reshape(Hkv, -1)[:, :S]
    for h in range(Hkv):
        have = set(kept[h].tolist())
        assert len(have) == S and {0, 1} <= have and set(range(n + steps - M, n + steps)) <= have
