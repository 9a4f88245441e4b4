"""The calls around steps over pages together, as a server makes them: map, norms and rotation, rows into pages, attention; in graphs, on
streams, and with tensors of other strides."""
import math

import pytest
import torch

from paper_2406_13035_amd import binding

from . import pages_ref
from . import serving_ref as ref

pytestmark = pytest.mark.gpu
BF16, I32 = torch.bfloat16, torch.int32
B, HQ, HKV, D, PAGE, CAP = 5, 8, 2, 128, 16, 12
EPS, BASE = 1e-6, 10000.0


class Server:
    """One layer of a server: tables, pools, and its calls for a turn of packed tokens."""

    def __init__(self, form, rows, seed=0):
        self.rows, n_pages = rows, B * CAP - 7
        g = torch.Generator().manual_seed(seed)
        i32 = lambda x: torch.tensor(x, dtype=I32, device="cuda:0")  # noqa: E731
        self.table = torch.full((B, CAP), -1, dtype=I32, device="cuda:0")
        self.lens, self.ring, self.state = i32([0] * B), torch.randperm(n_pages, generator=g).to(I32).cuda(), i32([0, n_pages])
        wide = D // 2 if form == "fp4" else D
        dt = torch.uint8 if form in ("fp4", "fp8") else BF16
        shape = (n_pages, HKV, PAGE)
        self.k, self.v = (torch.zeros((*shape, wide), dtype=dt, device="cuda:0") for _ in range(2))
        exps = (*shape, D // 32) if form == "fp4" else shape
        self.ke, self.ve = (torch.zeros(exps, dtype=torch.int8, device="cuda:0") if dt == torch.uint8 else None for _ in range(2))
        self.pages = binding.Pages(self.k, self.v, self.table, HQ, K_exp=self.ke, V_exp=self.ve)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(D, generator=g)).to(BF16).cuda() for _ in range(2))
        # what a turn is given, and gives
        self.change = i32([0] * B)
        self.qkv = torch.zeros((rows, HQ + 2 * HKV, D), dtype=BF16, device="cuda:0")
        self.first, self.slots = i32([0] * (B + 1)), torch.zeros(rows, dtype=torch.int64, device="cuda:0")
        self.positions, self.out = i32([0] * rows), torch.zeros((rows, HQ, D), dtype=BF16, device="cuda:0")
        self.form = form

    def turn(self):
        binding.d2o_pages_map(self.table, self.lens, self.change, self.ring, self.state, PAGE, first=self.first, slots=self.slots,
                              positions=self.positions)
        q, k, v = self.qkv[None, :, :HQ].transpose(1, 2), self.qkv[None, :, HQ:HQ + HKV].transpose(1, 2), self.qkv[:, HQ + HKV:]
        binding.d2o_qk_norm_rope(q, k, self.wq, self.wk, EPS, self.positions[None], rope_base=BASE, Q_out=q, K_out=k)
        self.pages.d2o_pages_put(self.qkv[:, HQ:HQ + HKV], v, self.slots)
        if self.form == "fp4":
            self.pages.d2o_pages_attend(self.qkv[:, :HQ], self.first, self.lens, self.out)
        else:
            self.pages.d2o_pages_step(self.qkv[:B, :HQ], None, None, self.lens, self.out[:B])


class Plain:
    """The same in 64 bits: lists of rows per sequence, rounded where the server's tensors are."""

    def __init__(self, s):
        self.k, self.v = [[] for _ in range(B)], [[] for _ in range(B)]
        self.wq, self.wk = s.wq.cpu(), s.wk.cpu()

    def turn(self, change, qkv, lens_before, lens_after, first, out):
        """Checks `out` [tokens, HQ, D]; the pool's capacity has been the walk's business (lens_after)."""
        for b in range(B):
            if change[b] < 0:
                self.k[b], self.v[b] = self.k[b][:lens_after[b]], self.v[b][:lens_after[b]]
            for i in range(first[b + 1] - first[b]):
                row = qkv[first[b] + i]
                pos = torch.tensor([[lens_before[b] + i]])
                q, tq = ref.norm_ref(row[None, :HQ, None], self.wq, EPS, D, pos, BASE)
                k, tk = ref.norm_ref(row[None, HQ:HQ + HKV, None], self.wk, EPS, D, pos, BASE)
                # (the server's own rounding of the rotated row to bf16 is taken over: what follows is about the attention)
                self.k[b].append(ref.rounded4(k[0, :, 0].to(BF16)))
                self.v[b].append(ref.rounded4(row[HQ + HKV:]))
                K, V = torch.stack(self.k[b]), torch.stack(self.v[b])
                for h in range(HQ):
                    p = torch.softmax(K[:, h // (HQ // HKV)] @ q[0, h, 0].to(BF16).double() / math.sqrt(D), 0)
                    want = p @ V[:, h // (HQ // HKV)]
                    err = (out[first[b] + i, h].double() - want).norm() / want.norm()
                    # half a step of bf16 (2^-8 of each element, at most), and what a q or k one step off in a few elements moves
                    assert float(err) < 2.0 ** -8 + 2.0 ** -7, (b, i, h, float(err))


def random_turns(n, seed):
    g = torch.Generator().manual_seed(seed)
    for t in range(n):
        change = torch.randint(1, 4, (B,), generator=g)
        if t == 0:
            change = torch.tensor([20, 1, 37, 0, 9])
        if t == 3:
            change[0], change[2] = -12, -1000
        if t == 5:
            change[1], change[3] = 70, 60
        yield change.tolist(), torch.randn((140, HQ + 2 * HKV, D), generator=g).to(BF16)


def test_turns_of_a_server_against_rows_in_lists():
    s = Server("fp4", 140)
    p = Plain(s)
    for change, qkv in random_turns(7, 1):
        before = s.lens.tolist()
        s.change.copy_(torch.tensor(change))
        s.qkv.copy_(qkv)
        s.turn()
        p.turn(change, qkv, before, s.lens.tolist(), s.first.tolist(), s.out.cpu())


@pytest.mark.parametrize("form", ["fp4", "fp8", "bf16"])
def test_turns_in_a_graph(form):
    """A captured turn, replayed with new inputs in its tensors and eager work between: every replay leaves what the eager call leaves."""
    turns = list(random_turns(7, 2)) if form == "fp4" else [([1] * B, torch.randn((140, HQ + 2 * HKV, D)).to(BF16)) for _ in range(6)]
    eager, graph = Server(form, 140), Server(form, 140)
    for s in (eager, graph):  # (a first turn outside, which also warms up)
        s.change.copy_(torch.tensor(turns[0][0]))
        s.qkv.copy_(turns[0][1])
        s.turn()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured, stream=side):
        graph.turn()
    for change, qkv in turns[1:]:
        for s in (eager, graph):
            s.change.copy_(torch.tensor(change))
            s.qkv.copy_(qkv)
        eager.turn()
        torch.cuda.synchronize()
        captured.replay()
        torch.randn(1000, device="cuda:0").sum().item()
        torch.cuda.synchronize()
        for x in ("table", "lens", "ring", "state", "first", "slots", "positions", "k", "v", "ke", "ve", "qkv", "out"):
            a, b = getattr(eager, x), getattr(graph, x)
            assert a is None or torch.equal(a, b), x


def test_calls_on_another_stream_than_the_tensors():
    a, b = Server("fp4", 140), Server("fp4", 140)
    side = torch.cuda.Stream()
    for change, qkv in random_turns(3, 4):
        for s in (a, b):
            s.change.copy_(torch.tensor(change))
            s.qkv.copy_(qkv)
        a.turn()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b.turn()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(a.out, b.out) and torch.equal(a.k, b.k) and torch.equal(a.lens, b.lens)


def test_two_calls_at_once_on_one_object():
    """Attention calls need no workspace of the object's: two on streams of their own may overlap."""
    t = ref.make_pages4(2, 2, 128, 64, 40, 3, score=False, pos=False)
    t = {k: None if x is None else x.cuda() for k, x in t.items()}
    pages = binding.Pages(t["k"], t["v"], t["table"], 8, K_exp=t["k_exp"], V_exp=t["v_exp"])
    lens, first = torch.tensor([2500, 2000], dtype=I32).cuda(), torch.tensor([0, 3, 40], dtype=I32).cuda()
    qs = [torch.randn((40, 8, 128), device="cuda:0").to(BF16) for _ in range(4)]
    want = [torch.zeros_like(q) for q in qs]
    for q, o in zip(qs, want):
        pages.d2o_pages_attend(q, first, lens, o)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    got = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for q, o, s in zip(qs, got, streams):
        with torch.cuda.stream(s):
            pages.d2o_pages_attend(q, first, lens, o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_one_token_by_attend_and_by_step():
    """A step without scores and an attention of one token each see the same entries."""
    t = ref.make_pages4(3, 2, 128, 16, 20, 7, score=False, pos=False)
    t = {k: None if x is None else x.cuda() for k, x in t.items()}
    pages = binding.Pages(t["k"], t["v"], t["table"], 6, K_exp=t["k_exp"], V_exp=t["v_exp"])
    lens = torch.tensor([300, 17, 1], dtype=I32).cuda()
    q = torch.randn((3, 6, 128), device="cuda:0").to(BF16)
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    for window, sink in ((0, 0), (40, 3)):
        pages.d2o_pages_step(q, None, None, lens, a, window=window, n_sink=sink)
        pages.d2o_pages_attend(q, torch.arange(4, dtype=I32).cuda(), lens, b, window=window, n_sink=sink)
        # both round once; sums in another order may fall to the other side of a step
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -7 * float(a.float().abs().max())


def test_pools_whose_offsets_pass_32_bits():
    """A pool of more than 4 GiB per tensor, the used pages at its end: rows put, read back and attended to there."""
    n_pages, page, Hkv = 160000, 64, 8
    k, v = (torch.zeros((n_pages, Hkv, page, 64), dtype=torch.uint8, device="cuda:0") for _ in range(2))
    ke, ve = (torch.zeros((n_pages, Hkv, page, 4), dtype=torch.int8, device="cuda:0") for _ in range(2))
    table = torch.tensor([[n_pages - 1, n_pages - 3, 5]], dtype=I32, device="cuda:0")
    pages = binding.Pages(k, v, table, Hkv, K_exp=ke, V_exp=ve)
    n = 150
    s = torch.arange(n)
    slots = (table.cpu()[0].long()[s // page] * page + s % page).cuda()
    K, V = (torch.randn((n, Hkv, 128), device="cuda:0").to(BF16) for _ in range(2))
    pages.d2o_pages_put(K, V, slots)
    Ko, Vo = torch.zeros_like(K), torch.zeros_like(V)
    pages.d2o_pages_get(slots, Ko, Vo)
    assert torch.equal(Ko.cpu().double(), ref.rounded4(K.cpu())) and torch.equal(Vo.cpu().double(), ref.rounded4(V.cpu()))
    q = torch.randn((40, Hkv, 128), device="cuda:0").to(BF16)
    out = torch.zeros_like(q)
    pages.d2o_pages_attend(q, torch.tensor([0, 40], dtype=I32).cuda(), torch.tensor([n], dtype=I32).cuda(), out)
    small = {"k": ref.rounded4(K.cpu()).transpose(0, 1)[None], "v": ref.rounded4(V.cpu()).transpose(0, 1)[None], "pos": None,
             "table": torch.zeros((1, 1), dtype=I32)}
    want, tol = ref.attend_ref(small, q.cpu(), [0, 40], [n], None, 0, 0, 1 << 20, torch.zeros(q.shape))
    assert bool(((out.cpu().double() - want).abs() <= tol).all())


def test_refused_by_the_binding():
    s = Server("fp4", 8)
    q = s.qkv[:, :HQ]
    for call in (lambda: s.pages.d2o_pages_attend(q, s.first[:-1], s.lens, s.out), lambda: s.pages.d2o_pages_attend(q, s.first, s.lens, s.out[:4]),
                 lambda: s.pages.d2o_pages_attend(q.float(), s.first, s.lens, s.out), lambda: s.pages.d2o_pages_attend(q, s.first, s.lens, s.out, window=-1),
                 lambda: s.pages.d2o_pages_put(q, q, s.slots), lambda: s.pages.d2o_pages_put(s.qkv[:, :2], s.qkv[:, :2], s.slots.int()),
                 lambda: s.pages.d2o_pages_get(s.slots, s.qkv[:, :2], s.qkv[:4, :2]),
                 lambda: binding.d2o_qk_norm_rope(q[None].transpose(1, 2), None, rot_dim=24), lambda: binding.d2o_qk_norm_rope(q[None].transpose(1, 2), None, eps=0.0),
                 lambda: binding.d2o_qk_norm_rope(q[None].transpose(1, 2), None, s.wq.float()),
                 lambda: binding.d2o_pages_map(s.table, s.lens, s.change, s.ring, s.state, 24, 8),
                 lambda: binding.d2o_pages_map(s.table, s.lens, s.change, s.ring, s.state, PAGE),
                 lambda: binding.d2o_pages_map(s.table, s.lens[:-1], s.change, s.ring, s.state, PAGE, 8),
                 lambda: binding.Pages(s.k, s.v, s.table, HQ), lambda: binding.Pages(s.k, s.v, s.table, HQ, K_exp=s.ke, V_exp=s.ve[..., 0].contiguous())):
        with pytest.raises(binding.D2OError):
            call()
    # nothing to do is no error
    s.pages.d2o_pages_attend(q[:0], s.first, s.lens, s.out[:0])
    s.pages.d2o_pages_put(s.qkv[:0, :2], s.qkv[:0, :2], s.slots[:0])
    s.pages.d2o_pages_get(s.slots[:0], s.qkv[:0, :2], s.qkv[:0, :2])
    torch.cuda.synchronize()
