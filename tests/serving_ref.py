"""Plain 64-bit forms, on the CPU, of what stands around a step over pages: 4-bit rows, norms with rotation, block tables and slots,
attention of several tokens per sequence; and the error bounds that the kernels' arithmetic allows."""
from __future__ import annotations

import math

import torch

from . import pages_ref as ref

GRID = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
NAN = -128


def encode4(x):
    """[.., d] to codes [.., d / 2] and powers of two [.., d / 32], by comparison with every code."""
    x = x.double().unflatten(-1, (-1, 32))
    broken = ~torch.isfinite(x).all(-1)
    x = torch.where(broken[..., None], torch.zeros_like(x), x)
    amax = x.abs().amax(-1)
    fr, ex = torch.frexp(amax)
    e = torch.where(amax > 0, torch.where(fr <= 0.75, ex - 3, ex - 2).clamp(-120, 125), torch.zeros_like(ex))
    a = torch.ldexp(x, -e[..., None]).abs()
    off = (a[..., None] - GRID).abs()
    # the nearest; among two as near the even code, which is the first of a sort by oddness
    order = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[off[..., order].argmin(-1)]
    code = torch.where(torch.signbit(x), code + 8, code).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(broken, torch.full_like(e, NAN), e).to(torch.int8)


def decode4(codes, e):
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = torch.where(both >= 8, -GRID[both % 8], GRID[both % 8]).unflatten(-1, (-1, 32))
    v = torch.ldexp(v, e[..., None].int())
    return torch.where((e == NAN)[..., None], torch.full_like(v, math.nan), v).flatten(-2)


def rounded4(x):
    return decode4(*encode4(x))


def make_pages4(batch, kv_heads, d, page, per_seq, seed, order="pool", score=True, pos=True, spare=3, scale=1.0):
    """As pages_ref.make_pages, with rows of 4 bits whose blocks differ in size."""
    t = ref.make_pages(batch, kv_heads, d, page, per_seq, torch.float32, seed, False, order, score, pos, spare)
    g = torch.Generator().manual_seed(seed + 1)
    for x in ("k", "v"):
        size = torch.exp2(torch.randint(-2, 3, (*t[x].shape[:3], d // 32, 1), generator=g).float())
        codes, t[x + "_exp"] = encode4((t[x].unflatten(-1, (-1, 32)) * size * scale).flatten(-2).to(torch.bfloat16))
        t[x] = codes.transpose(1, 2).contiguous().transpose(1, 2) if order == "token" else codes.contiguous()
        t[x + "_exp"] = t[x + "_exp"].contiguous()
    return t


def values(t):
    """The same tables with rows as 64-bit values, for the forms that know no codes."""
    return {**t, "k": decode4(t["k"], t["k_exp"]), "v": decode4(t["v"], t["v_exp"]), "k_exp": None, "v_exp": None}


def step_ref4(t, q, k_new, v_new, lens, positions, window, n_sink, max_len):
    """pages_ref.step_ref over 4-bit rows (new rows as they are encoded); weights enter P V as two bf16 terms: off by 2^-8 * 2^-8 of
    themselves, so the output by that much of the same mean of magnitudes."""
    kn, vn = (None if x is None else rounded4(x) for x in (k_new, v_new))
    w = values(t)
    out, tol, new, add, add_tol = ref.step_ref(w, q, kn, vn, lens, positions, window, n_sink, max_len, torch.bfloat16)
    big = ref.step_ref({**w, "v": w["v"].abs()}, q, kn, None if vn is None else vn.abs(), lens, positions, window, n_sink, max_len,
                       torch.bfloat16)[0]
    return out, tol + 2.0 ** -16 * big, new, add, add_tol


def attend_ref(w, q, first, lens, positions, window, n_sink, max_len, before):
    """(out, bound) of d2o_pages_attend in 64 bits over the values `w`; rows of no token as in `before`."""
    n_tokens, Hq, d = q.shape
    Hkv = w["k"].shape[1]
    G = Hq // Hkv
    out, tol = before.double().clone(), torch.zeros(before.shape, dtype=torch.float64)
    for b in range(len(lens)):
        q0, q1 = (min(max(int(x), 0), n_tokens) for x in first[b:b + 2])
        m, n = q1 - q0, min(int(lens[b]), max_len)
        for i in range(max(m, 0)):
            mine = n - m + i
            out[q0 + i] = 0.0
            if mine < 0:
                continue
            P = int(positions[q0 + i]) if positions is not None else mine
            p, r = ref.entries(w, b, mine + 1)
            s = torch.arange(mine + 1)[p >= 0]
            p, r = p[s], r[s]
            for h in range(Hkv):
                at = w["pos"][p, h, r].long() if w["pos"] is not None else s
                seen = (at > P - window) | (at < n_sink) if window else torch.ones(len(s), dtype=torch.bool)
                if not seen.any():
                    continue
                k, v = w["k"][p[seen], h, r[seen]], w["v"][p[seen], h, r[seen]]
                qq = q[q0 + i, h * G:(h + 1) * G].double()
                if not torch.isfinite(k).all():
                    out[q0 + i, h * G:(h + 1) * G] = math.nan
                    continue
                every = torch.ones((G, len(k)), dtype=torch.bool)
                o, pr = ref.attend64(qq, k, v, every)
                out[q0 + i, h * G:(h + 1) * G] = o
                fine = torch.nan_to_num(v)
                tol[q0 + i, h * G:(h + 1) * G] = ref.bound(qq, k, fine, every, torch.nan_to_num(o), pr, torch.bfloat16, False) + (
                    2.0 ** -16 * (pr @ fine.abs()))
    return out, tol


def norm_ref(x, w, eps, rot, positions, base):
    """(y, bound) of one of Q and K [B, H, n, d]; positions [B, n].

    The sum of d squares and the root: (d / 2 + 3) half steps of 2^-24, two products and the rotation's two products and sum four more;
    the angle: a fraction of a turn rounded to 2^-25 of its half (2^-23 of a radian), sine and cosine two steps, the position's
    product with a 64-bit factor 2^-52 of itself; the result rounded once."""
    y = x.double()
    y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    y = y * w.double() if w is not None else y
    half = rot // 2
    c = torch.arange(half, dtype=torch.float64)
    angle = positions.double()[:, None, :, None] * torch.exp(-2.0 * c / max(rot, 1) * math.log(base))
    a, b, rest = y[..., :half], y[..., half:rot], y[..., rot:]
    out = torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin(), rest], -1)
    mag = torch.cat([a.abs() + b.abs(), a.abs() + b.abs(), rest.abs()], -1)
    far = positions.double().abs()[:, None, :, None]
    tol = mag * ((x.shape[-1] / 2 + 9) * 2.0 ** -24 + 2.0 ** -22 + far * 2.0 ** -51) + out.abs() * ref.HALF_STEP[x.dtype] + 1e-38
    return out, tol


def map_ref(table, lens, change, ring, state, page, rows):
    """d2o_pages_map as a walk from sequence to sequence; all arguments lists."""
    cap, n_pages = len(table[0]), len(ring)
    head, count = state
    pages = lambda n: -(-n // page)  # noqa: E731
    table, ring = [list(t) for t in table], list(ring)
    after, first, slots, positions = [], [0], [], []
    tokens = wanted = taken = 0
    tail = []
    for b, (n, c) in enumerate(zip(lens, change)):
        n = min(max(n, 0), cap * page)
        gain, loss = max(c, 0), min(max(-c, 0), n)
        if n + gain > cap * page:
            gain = 0
        need = pages(n + gain) - pages(n)
        tokens, wanted = tokens + gain, wanted + need
        if tokens > rows or (need and wanted > count):
            gain = need = 0
        for i in range(need):
            table[b][pages(n) + i] = ring[(head + taken) % n_pages]
            taken += 1
        tail += [table[b][i] for i in range(pages(n - loss), pages(n))] if loss else []
        for p in range(n, n + gain):
            at = table[b][p // page]
            slots.append(at * page + p % page if 0 <= at < n_pages else -1)
            positions.append(p)
        after.append(n + gain - loss)
        first.append(len(slots))
    tail = tail[:n_pages - count]
    for i, p in enumerate(tail):
        ring[(head + count + i) % n_pages] = p
    idle = rows - len(slots)
    return table, after, ring, [(head + taken) % n_pages, count - taken + len(tail)], first, slots + [-1] * idle, positions + [0] * idle
