"""Windowed prompt attention with sink tokens against its 64-bit form, at tile edges, odd sizes, strides and values
where it can go wrong."""
import math

import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def inputs(dtype, B, Hq, Hkv, n, d, seed=0, qscale=1.5):
    g = torch.Generator().manual_seed(1000 + seed)
    r = lambda h, s=1.0: (torch.randn((B, h, n, d), generator=g) * s).to(dtype)  # noqa: E731
    return r(Hq, qscale), r(Hkv), r(Hkv)


def check(Q, K, V, O, window, n_sink, lens=None, heads=None):
    """O (on the CPU) against the definition; rows behind a sequence's end are not looked at here, nor heads other than `heads`."""
    B, Hq, n, d = Q.shape
    G = Hq // K.shape[1]
    for b in range(B):
        m = n if lens is None else int(lens[b])
        if m == 0:
            continue
        seen = ref.window_seen(m, window, n_sink)
        for h in heads if heads is not None else range(Hq):
            q, k, v = (x[b, i, :m].double() for x, i in ((Q, h), (K, h // G), (V, h // G)))
            o, p = ref.attend64(q, k, v, seen)
            got = O[b, h, :m].double()
            fine = torch.isfinite(o)
            assert torch.equal(torch.isfinite(got), fine), (b, h)
            assert torch.equal(got.isnan(), o.isnan()) and torch.equal(got[got.isinf()], o[o.isinf()])
            # (columns without an infinity or NaN: these have no bound)
            vf = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
            tol = ref.bound(q, k, vf, seen, torch.where(fine, o, torch.zeros_like(o)), p, Q.dtype, Q.dtype == BF16)
            err = torch.where(fine, (got - o).abs(), torch.zeros_like(o))
            assert bool((err <= tol).all()), (b, h, float((err / tol).max()))


def run(Q, K, V, window, n_sink, lens=None, O=None):
    dev = "cuda:0"
    O = binding.d2o_window_attend(Q.to(dev), K.to(dev), V.to(dev), window, n_sink, None if lens is None else lens.to(dev), O)
    torch.cuda.synchronize()
    return O.cpu()


SIZES = [  # B, Hq, Hkv, n, window, n_sink
    (1, 1, 1, 1, 0, 0), (1, 2, 1, 2, 1, 0), (2, 4, 2, 5, 3, 1), (1, 4, 4, 31, 8, 2), (1, 3, 1, 33, 1, 0),
    (1, 4, 1, 63, 17, 4), (1, 2, 2, 64, 64, 0), (1, 8, 1, 65, 33, 40), (1, 16, 1, 96, 0, 0), (2, 6, 2, 127, 64, 3),
    (1, 2, 2, 128, 63, 64), (1, 2, 1, 129, 65, 65), (1, 5, 5, 200, 100, 150), (1, 4, 2, 257, 129, 1), (1, 2, 2, 256, 300, 7),
    (1, 1, 1, 513, 2, 130), (1, 2, 1, 700, 350, 0), (1, 2, 2, 641, 0, 4), (3, 2, 1, 300, 1, 1), (1, 2, 2, 1100, 64, 4),
    (1, 1, 1, 2000, 1031, 77),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "b%d_q%d_kv%d_n%d_w%d_t%d" % s)
def test_window_attend(dtype, d, size):
    B, Hq, Hkv, n, window, n_sink = size
    Q, K, V = inputs(dtype, B, Hq, Hkv, n, d, seed=n)
    check(Q, K, V, run(Q, K, V, window, n_sink), window, n_sink)


@pytest.mark.parametrize("dtype,d,heads,n,window,n_sink,lens", [
    (BF16, 128, (64, 16), 1111, 1029, 5, None), (BF16, 128, (60, 60), 1100, 0, 0, None), (BF16, 128, (60, 10), 1090, 1088, 70, [1090, 777]),
    (BF16, 128, (64, 8), 1200, 1150, 4, [1200, 65]), (BF16, 128, (60, 15), 700, 300, 4, None), (BF16, 128, (72, 24), 650, 33, 65, [640, 3]),
    (BF16, 64, (60, 60), 700, 129, 4, None), (BF16, 64, (64, 8), 1111, 1029, 0, [1111, 1, 500]), (F32, 64, (24, 4), 700, 100, 4, None),
    (F32, 128, (32, 32), 600, 0, 0, [600, 333]), (F32, 128, (16, 2), 1100, 257, 33, [1100, 64]), (F32, 64, (40, 10), 450, 1, 1, None),
], ids=str)
def test_many_heads(dtype, d, heads, n, window, n_sink, lens):
    """Enough rows for every kernel's larger blocks and for several heads of a group in one; a few values are not finite."""
    Q, K, V = inputs(dtype, len(lens) if lens else 1, *heads, n, d, seed=n)
    for h, j in ((0, 3), (heads[1] - 1, 100), (heads[1] - 1, n // 2)):
        V[0, h, j, j % d] = math.inf
    lens = torch.tensor(lens, dtype=torch.int32) if lens else None
    got = run(Q, K, V, window, n_sink, lens)
    G = heads[0] // heads[1]
    check(Q, K, V, got, window, n_sink, lens, heads=sorted({0, G - 1, heads[0] // 2, heads[0] - G, heads[0] - 1}))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_padded_batch(dtype):
    """Sequences of different lengths, one of them empty: their rows are right, the rows behind them untouched, and what lies
    in the padding - infinities and NaN - takes no part."""
    B, Hq, Hkv, n, d = 5, 4, 2, 300, 128
    lens = torch.tensor([300, 0, 1, 130, 257], dtype=torch.int32)
    Q, K, V = inputs(dtype, B, Hq, Hkv, n, d)
    for b in range(B):
        K[b, :, lens[b]:] = math.nan
        V[b, :, lens[b]:] = math.inf
        Q[b, :, lens[b]:] = math.nan
    O = torch.full(Q.shape, 7.0, dtype=dtype, device="cuda:0")
    got = run(Q, K, V, 100, 3, lens, O)
    check(Q, K, V, got, 100, 3, lens)
    for b in range(B):
        assert bool((got[b, :, lens[b]:] == 7.0).all())
    fresh = run(Q, K, V, 100, 3, lens)
    for b in range(B):
        assert torch.equal(fresh[b, :, :lens[b]], got[b, :, :lens[b]]) and bool((fresh[b, :, lens[b]:] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_lengths_beyond_the_tensor_are_cut(dtype):
    Q, K, V = inputs(dtype, 2, 2, 1, 70, 64)
    got = run(Q, K, V, 20, 1, torch.tensor([1 << 30, -5], dtype=torch.int32))
    check(Q, K, V, got, 20, 1, [70, 0])
    assert bool((got[1] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_strided_views(dtype):
    """Token-major tensors with padded rows and heads in the middle of a wider one."""
    B, Hq, Hkv, n, d = 2, 4, 2, 150, 64
    Q, K, V = inputs(dtype, B, Hq, Hkv, n, d)
    wide = torch.zeros((B, n, Hq + 2 * Hkv + 1, d + 16), dtype=dtype, device="cuda:0")
    q, k, v = wide[:, :, :Hq, :d], wide[:, :, Hq:Hq + Hkv, :d], wide[:, :, Hq + Hkv:Hq + 2 * Hkv, :d]
    for x, y in ((q, Q), (k, K), (v, V)):
        x.copy_(y.transpose(1, 2))
    out = torch.full((B, n, Hq, d + 16), 7.0, dtype=dtype, device="cuda:0")
    binding.d2o_window_attend(q.transpose(1, 2), k.transpose(1, 2), v.transpose(1, 2), 40, 5, O=out[..., :d].transpose(1, 2))
    want = run(Q, K, V, 40, 5)
    assert torch.equal(out[..., :d].transpose(1, 2).cpu(), want)
    assert bool((out[..., d:] == 7.0).all())


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_values_that_are_not_finite_reach_only_who_sees_them(dtype, value):
    Q, K, V = inputs(dtype, 1, 2, 1, 300, 64)
    for j, c in ((0, 3), (70, 5), (128, 0), (200, 63), (255, 17), (299, 9)):
        V[0, 0, j, c] = value
    check(Q, K, V, run(Q, K, V, 50, 2), 50, 2)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_both_infinities_of_a_column_cancel_to_nan_where_both_are_seen(dtype):
    Q, K, V = inputs(dtype, 1, 1, 1, 200, 128)
    V[0, 0, 100, 7], V[0, 0, 130, 7] = math.inf, -math.inf
    check(Q, K, V, run(Q, K, V, 64, 0), 64, 0)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_keys_that_are_not_finite_reach_only_who_sees_them(dtype):
    """A NaN key makes the rows that see it NaN, whole; the others are as if it were any other key."""
    Q, K, V = inputs(dtype, 1, 1, 1, 260, 64)
    K[0, 0, 100] = math.nan
    got = run(Q, K, V, 40, 0)
    hit = torch.zeros(260, dtype=torch.bool)
    hit[100:140] = True
    assert bool(got[0, 0, hit].isnan().all()) and bool(torch.isfinite(got[0, 0, ~hit]).all())
    K[0, 0, 100] = 0.0
    clean = run(Q, K, V, 40, 0)
    assert torch.equal(got[0, 0, ~hit], clean[0, 0, ~hit])


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e6, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_values_of_any_magnitude(dtype, scale):
    Q, K, V = inputs(dtype, 1, 2, 2, 200, 128)
    V = (V.float() * scale).to(dtype)
    check(Q, K, V, run(Q, K, V, 70, 4), 70, 4)


def test_values_whose_magnitude_changes_along_the_prompt():
    """Every eighth token's values are larger or smaller by powers of two: each output is dominated by the large ones it sees."""
    Q, K, V = inputs(BF16, 1, 2, 1, 400, 64)
    e = torch.randint(-40, 40, (50,), generator=torch.Generator().manual_seed(5)).repeat_interleave(8)
    V = torch.ldexp(V.float(), e[None, None, :, None]).to(BF16)
    check(Q, K, V, run(Q, K, V, 60, 3), 60, 3)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_sharp_and_flat_attention(dtype):
    """Logits in the hundreds (one key takes all), and all equal (the mean of what is seen)."""
    Q, K, V = inputs(dtype, 1, 2, 1, 260, 128, qscale=60.0)
    check(Q, K, V, run(Q, K, V, 90, 2), 90, 2)
    Q = torch.zeros_like(Q)
    check(Q, K, V, run(Q, K, V, 90, 2), 90, 2)


@pytest.mark.parametrize("total", [14, 20, 27, 40, 115])
@pytest.mark.parametrize("dtype,d,heads,n,window,n_sink", [
    (F32, 64, (2, 1), 300, 90, 2), (F32, 128, (24, 4), 700, 300, 70), (BF16, 64, (2, 1), 300, 90, 2), (BF16, 128, (2, 1), 300, 0, 0),
    (BF16, 64, (60, 60), 700, 300, 4), (BF16, 128, (60, 60), 700, 300, 70), (BF16, 128, (64, 16), 1111, 1029, 5),
], ids=str)
def test_logits_of_any_size(dtype, d, heads, n, window, n_sink, total):
    """Logits of up to 255 times 2^total: products of one pair of numbers, so exact in fp32, and steps of 2^total / sqrt(d) apart, so a
    row attends to its highest key, or to those that share its value, alone.  Rows in turn: of such logits, of their negatives, of all-zero
    ones and of small ones.  A wavefront holds all four, and meets the huge ones in any tile of its window."""
    g = torch.Generator().manual_seed(total)
    Q, K = torch.zeros((1, heads[0], n, d)), torch.zeros((1, heads[1], n, d))
    K[0, :, :, 0] = torch.randint(1, 256, (heads[1], n), generator=g).float() * 2.0 ** (total // 2)
    Q[0, :, :, 0] = torch.tensor([2.0 ** (total - total // 2), -2.0 ** (total - total // 2), 0.0, 2.0 ** -(total // 2)]).repeat(n)[:n]
    V = torch.randn((1, heads[1], n, d), generator=g).to(dtype)
    Q, K, seen = Q.to(dtype), K.to(dtype), ref.window_seen(n, window, n_sink)
    O = run(Q, K, V, window, n_sink)
    # the small rows' logits, at most 32, rounded three times, all of them scaled and their exponentials rounded: in the sum and in the normaliser
    rel = 2 * (32 * 3 * 2.0 ** -24 + 2.0 ** -22 + n * 2.0 ** -24) + (2.0 ** -11 if dtype == BF16 else 0)
    for h in (0, heads[0] // 2, heads[0] - 1):
        q, k, v = (x[0, i].double() for x, i in ((Q, h), (K, h * heads[1] // heads[0]), (V, h * heads[1] // heads[0])))
        o, p = ref.attend64(q, k, v, seen)
        tol = p @ v.abs() * rel + o.abs() * ref.HALF_STEP[dtype] + (float(v.abs().max()) * n * 2.0 ** -36 if dtype == BF16 else 0)
        err = (O[0, h].double() - o).abs()
        assert bool((err <= tol).all()), (h, float((err / tol).max()))


@pytest.mark.parametrize("start", [-200, -7, 4096, 1 << 20])
@pytest.mark.parametrize("dtype,heads,window", [(F32, 2, 0), (BF16, 2, 0), (BF16, 2, 200), (BF16, 60, 200)], ids=str)
def test_large_logits_that_grow_along_the_prompt(dtype, heads, window, start):
    """Logits near 5814543, whose exponents lie near 2^20, and beyond, exact in fp32: 20 more every 64 tokens, where the tokens before still weigh."""
    n, d = 1280, 64
    Q, K, V = inputs(dtype, 1, heads, heads, n, d)
    Q[:], K[:] = 0, 0
    Q[..., :4] = 2048
    Q[..., 4:7] = 1
    for c, x in enumerate((2048, 768, 23, max(start, 0) / 2048, 271 - 256 + min(start, 0), 256)):
        K[..., c] = x
    K[..., 6] = (torch.arange(n) // 64 * 20).to(dtype)
    assert float(Q[0, 0, 0].double() @ K[0, 0, 64].double()) == 5814543 + start + 20
    O, seen = run(Q, K, V, window, 0), ref.window_seen(n, window, 0)
    # an exponent of up to 2^21 is rounded to fp32: by 2^-4 at most, in the sum and in the normaliser; the rest is below 2^-9
    rel = 2 * (2.0 ** 2.0 ** -4 - 1) + 2.0 ** -9
    for h in (0, heads - 1):
        q, k, v = (x[0, h].double() for x in (Q, K, V))
        o, p = ref.attend64(q, k, v, seen)
        err = (O[0, h].double() - o).abs()
        tol = p @ v.abs() * rel + o.abs() * ref.HALF_STEP[dtype]
        assert bool((err <= tol).all()), (h, float((err / tol).max()))


@pytest.mark.parametrize("scale", [1e-10, 1e-6, 1.0, 1e10])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_runs_of_tokens_whose_values_are_zero(dtype, scale):
    """They take their share of the weights and change nothing about the accuracy of the others."""
    Q, K, V = inputs(dtype, 1, 2, 1, 500, 64)
    V = (V.float() * scale).to(dtype)
    V[:, :, 64:128] = 0
    V[:, :, 250:400] = 0
    check(Q, K, V, run(Q, K, V, 150, 3), 150, 3)
    V[:, :, :64] = 0
    check(Q, K, V, run(Q, K, V, 0, 0), 0, 0)


def test_two_runs_and_another_stream_give_the_same_bits():
    Q, K, V = (x.cuda() for x in inputs(BF16, 2, 8, 2, 900, 128))
    first = binding.d2o_window_attend(Q, K, V, 300, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = binding.d2o_window_attend(Q, K, V, 300, 4)
    s.synchronize()
    assert torch.equal(first, second)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_captured_and_replayed(dtype):
    Q, K, V = (x.cuda() for x in inputs(dtype, 1, 4, 2, 333, 128))
    lens = torch.tensor([333], dtype=torch.int32, device="cuda:0")
    O = torch.zeros_like(Q)
    binding.d2o_window_attend(Q, K, V, 77, 4, lens, O)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.d2o_window_attend(Q, K, V, 77, 4, lens, O)
    for seed, m in ((1, 333), (2, 200), (3, 1)):
        for x, y in zip((Q, K, V), inputs(dtype, 1, 4, 2, 333, 128, seed)):
            x.copy_(y)
        lens.fill_(m)
        O.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = binding.d2o_window_attend(Q, K, V, 77, 4, lens)
        assert torch.equal(O, want) and bool((O[:, :, :m] != 0).any())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_the_largest_window_and_number_of_first_tokens(dtype):
    Q, K, V = inputs(dtype, 1, 2, 1, 200, 64)
    want = run(Q, K, V, 0, 0)
    check(Q, K, V, want, 0, 0)
    for window, n_sink in ((0x7FFFFFFF, 0), (200, 5), (0x7FFFFFFF, 0x7FFFFFFF)):
        assert torch.equal(run(Q, K, V, window, n_sink), want)
    # every token a first one: the window adds nothing (the order of the sums may differ)
    check(Q, K, V, run(Q, K, V, 1, 0x7FFFFFFF), 1, 0x7FFFFFFF)


@pytest.mark.parametrize("n,heads", [(150, 4), (150, 300)], ids=["few", "many"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_offsets_beyond_32_bits(dtype, n, heads):
    """Rows millions of elements apart: the last ones lie more than 4 GiB behind the first."""
    d, step = 64, (1 << 24) - 64
    Q, K, V = inputs(dtype, 1, heads, heads, n, d)
    big = torch.empty(step * n + 2 * heads * d, dtype=dtype, device="cuda:0")
    k, v = (big.as_strided((1, heads, n, d), (0, d, step, 1), at) for at in (0, heads * d))
    k.copy_(K), v.copy_(V)
    O = binding.d2o_window_attend(Q.cuda(), k, v, 60, 3)
    assert torch.equal(O.cpu(), run(Q, K, V, 60, 3))
    with pytest.raises(binding.D2OError):
        binding.d2o_window_attend(Q[:, :, 1:].cuda(), big.as_strided((1, heads, n - 1, d), (0, d, 1 << 24, 1)), v[:, :, 1:], 60, 3)


def test_output_in_the_place_of_the_queries():
    for dtype in (F32, BF16):
        Q, K, V = (x.cuda() for x in inputs(dtype, 1, 4, 2, 700, 64))
        want = binding.d2o_window_attend(Q, K, V, 90, 2)
        assert binding.d2o_window_attend(Q, K, V, 90, 2, O=Q) is Q and torch.equal(Q, want)


def test_wrong_arguments_are_refused():
    Q, K, V = (x.cuda() for x in inputs(BF16, 2, 4, 2, 10, 64))
    bad = [
        lambda: binding.d2o_window_attend(Q.cpu(), K, V, 4),
        lambda: binding.d2o_window_attend(Q, K.float(), V, 4),
        lambda: binding.d2o_window_attend(Q, K, V[:, :, :9], 4),
        lambda: binding.d2o_window_attend(Q, K[:, :1].expand(2, 3, 10, 64), V[:, :1].expand(2, 3, 10, 64), 4),
        lambda: binding.d2o_window_attend(Q, K, V, -1),
        lambda: binding.d2o_window_attend(Q, K, V, 4, -1),
        lambda: binding.d2o_window_attend(Q, K, V, 1 << 32),
        lambda: binding.d2o_window_attend(Q, K, V, 4, lens=torch.tensor([1, 2], device="cuda:0")),
        lambda: binding.d2o_window_attend(Q, K, V, 4, O=torch.empty(2, 4, 10, 64, device="cuda:0")),
        lambda: binding.d2o_window_attend(Q[..., :32], K[..., :32], V[..., :32], 4),
        lambda: binding.d2o_window_attend(Q.transpose(2, 3), K.transpose(2, 3), V.transpose(2, 3), 4),
    ]
    for call in bad:
        with pytest.raises(binding.D2OError):
            call()
