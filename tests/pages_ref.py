"""Plain 64-bit forms of windowed prompt attention and of the calls on caches in pages, on the CPU, and the error bounds
that the arithmetic of the kernels allows."""
from __future__ import annotations

import math

import numpy as np
import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def attend64(q, k, v, seen):
    """q [.., m, d], k, v [.., n, d] in float64, seen [.., m, n].  (o, p, bound factors): rows that see nothing are zero.
    V counts only where it is seen: a masked infinity or NaN takes no part."""
    s = q @ k.transpose(-1, -2) / math.sqrt(q.shape[-1])
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isneginf(m), torch.zeros_like(m), m)), torch.zeros_like(s))
    total = p.sum(-1, keepdim=True)
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    if bool(torch.isfinite(v).all()):
        return p @ v, p
    o = torch.zeros(p.shape[:-1] + v.shape[-1:], dtype=torch.float64)
    for j in range(v.shape[-2]):
        row = p[..., :, j, None] * v[..., j, None, :]
        o = o + torch.where(seen[..., :, j, None], row, torch.zeros_like(row))
    return o, p


def bound(q, k, v, seen, o, p, out_dtype, half_terms):
    """Largest error of an output element.  The logits are fp32 sums of d products (error at most (d + 3) half steps of
    2^-24 times the sum of the magnitudes, in units of the exponent), the exponentials fp32 (2^-22 with the argument's
    rounding), the sums over n terms fp32; `half_terms`: the probabilities enter the product with V in fp16
    (2^-11 each, and an absolute 2^-36 of the largest for those that leave its normal range), else in fp32.  Both the numerator
    and the normaliser have the exponentials' errors: twice.  The output is rounded to its type once."""
    d, n = q.shape[-1], k.shape[-2]
    mag = (q.abs() @ k.abs().transpose(-1, -2)) / math.sqrt(d)
    mag = torch.where(seen, mag, torch.zeros_like(mag)).amax(-1, keepdim=True)
    rel = 2 * (mag * (d + 3) * 2.0 ** -24 + mag * 2.0 ** -22 + 2.0 ** -22 + n * 2.0 ** -24)
    if half_terms:
        rel = rel + 2.0 ** -11
    av = p @ v.abs()
    extra = v.abs().amax(-2, keepdim=True) * n * 2.0 ** -36 if half_terms else 0.0
    return av * rel + extra + o.abs() * HALF_STEP[out_dtype] + 1e-38


def window_seen(n, window, n_sink):
    i, j = torch.arange(n)[:, None], torch.arange(n)[None, :]
    return (j <= i) & ((j > i - (window or n)) | (j < n_sink))


# ---- pages --------------------------------------------------------------------------------

def make_pages(batch, kv_heads, d, page, per_seq, dtype, seed, fp8=False, order="pool", score=True, pos=True, spare=3):
    """Tensors of a pool with random pages handed out in random order; `order` "token": rows of a page lie [row][head]."""
    g = torch.Generator().manual_seed(seed)
    n_pages = batch * per_seq + spare
    shape = (n_pages, kv_heads, page, d)
    t = {}
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g).to(torch.bfloat16 if fp8 else dtype)
        if fp8:
            x, t[name + "_exp"] = encode(x)
        if order == "token":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        t[name] = x
    t.setdefault("k_exp", None)
    t.setdefault("v_exp", None)
    t["score"] = torch.rand(shape[:3], generator=g) if score else None
    t["pos"] = torch.randint(0, 1 << 20, shape[:3], generator=g, dtype=torch.int32) if pos else None
    t["table"] = torch.randperm(n_pages, generator=g)[:batch * per_seq].view(batch, per_seq).to(torch.int32).contiguous()
    return t


def encode(x):
    """Codes of the 8-bit float E4M3 and a power of two per row: the smallest that brings the row to 448 or below."""
    x = x.double()
    amax = x.abs().amax(-1)
    fr, ex = torch.frexp(amax)
    e = torch.where(amax > 0, torch.clamp(torch.where(fr <= 0.875, ex - 9, ex - 8), min=-120), torch.zeros_like(ex))
    y = torch.ldexp(x, -e[..., None]).float().to(torch.float8_e4m3fn)  # (exact before the rounding to eight bits)
    codes = y.view(torch.uint8)
    return torch.where(codes == 0x80, torch.zeros_like(codes), codes), e.to(torch.int8)


def rows64(pool, exps, page, h, r):
    x = pool[page, h, r]
    if exps is None:
        return x.double()
    return torch.ldexp(x.view(torch.float8_e4m3fn).double(), exps[page, h, r].int()[..., None])


def entries(t, b, n):
    """(page, row) of entries 0 .. n-1 of sequence b; page -1 where the table names none."""
    page = t["k"].shape[2]
    s = torch.arange(n)
    p = t["table"][b].long()[s // page]
    p = torch.where((p >= 0) & (p < t["k"].shape[0]), p, torch.full_like(p, -1))
    return p, s % page


def score_order(score, pos, guard, present):
    """Entries from the one kept first to the one given up first."""
    s = np.where(np.isnan(score), np.inf, score.astype(np.float64))
    nan = np.isnan(score)
    n = len(s)
    return np.array(sorted(range(n), key=lambda i: (not present[i], not guard[i], not nan[i], -s[i], pos[i], i)), dtype=np.int64)


def evict_ref(t, lens, budget, recent, n_sink):
    """The tensors after d2o_pages_evict, as new ones."""
    out = {k: (None if x is None else x.clone()) for k, x in t.items()}
    names = [x for x in ("k", "v", "k_exp", "v_exp", "score", "pos") if t[x] is not None]
    for b, n in enumerate(lens):
        if n <= budget:
            continue
        p, r = entries(t, b, n)
        for h in range(t["k"].shape[1]):
            present = (p >= 0).numpy()
            pc = p.clamp(min=0)
            score, pos = t["score"][pc, h, r].numpy(), t["pos"][pc, h, r].numpy().astype(np.int64)
            newest = pos[present].max() if present.any() else 0
            guard = present & ((pos < n_sink) | (pos > newest - recent))
            keep = np.zeros(n, bool)
            keep[score_order(score, pos, guard, present)[:budget]] = True
            holes = [s for s in range(budget) if not keep[s] and present[s]]
            late = [s for s in range(budget, n) if keep[s] and present[s]]
            for to, src in zip(holes, late):
                for x in names:
                    out[x][p[to], h, r[to]] = t[x][p[src], h, r[src]]
    return out


def fill_ref(t, K, V, lens, scores, budget, recent, n_sink):
    """The tensors after d2o_pages_fill, as new ones."""
    out = {k: (None if x is None else x.clone()) for k, x in t.items()}
    fp8 = t["k_exp"] is not None
    for b, n in enumerate(lens):
        kept = min(n, budget)
        if kept == 0:
            continue
        p, r = entries(t, b, kept)
        for h in range(t["k"].shape[1]):
            if n > budget:
                pos = np.arange(n)
                guard = (pos < n_sink) | (pos >= n - recent)
                src = np.sort(score_order(scores[b, h, :n].numpy(), pos, guard, np.ones(n, bool))[:budget])
            else:
                src = np.arange(n)
            ok = p >= 0
            src = torch.from_numpy(src)[ok]
            at = (p[ok], h, r[ok])
            for name, x in (("k", K), ("v", V)):
                if fp8:
                    out[name][at], out[name + "_exp"][at] = encode(x[b, h, src])
                else:
                    out[name][at] = x[b, h, src]
            if t["score"] is not None:
                out["score"][at] = scores[b, h, src] if scores is not None else 0.0
            if t["pos"] is not None:
                out["pos"][at] = src.to(torch.int32)
    return out


def step_ref(t, q, k_new, v_new, lens, positions, window, n_sink, max_len, out_dtype):
    """(out, bound, tensors with the new rows, added scores, their bound) of d2o_pages_step in 64 bits."""
    new = {k: (None if x is None else x.clone()) for k, x in t.items()}
    B, Hq, d = q.shape
    Hkv = t["k"].shape[1]
    G = Hq // Hkv
    out, tol = torch.zeros((B, Hq, d), dtype=torch.float64), torch.zeros((B, Hq, d), dtype=torch.float64)
    add = torch.zeros(t["k"].shape[:3], dtype=torch.float64)
    add_tol = torch.zeros_like(add)
    for b in range(B):
        n = min(int(lens[b]), max_len)
        if n <= 0:
            continue
        P = int(positions[b]) if positions is not None else n - 1
        p, r = entries(t, b, n)
        if k_new is not None and lens[b] <= max_len and p[n - 1] >= 0:
            at = (p[n - 1], slice(None), r[n - 1])
            for name, x in (("k", k_new), ("v", v_new)):
                if t[name + "_exp"] is not None:
                    new[name][at], new[name + "_exp"][at] = encode(x[b])
                else:
                    new[name][at] = x[b]
            if t["score"] is not None:
                new["score"][at] = 0.0
            if t["pos"] is not None:
                new["pos"][at] = P
        ok = p >= 0
        s = torch.arange(n)[ok]
        p, r = p[ok], r[ok]
        for h in range(Hkv):
            at = new["pos"][p, h, r].long() if t["pos"] is not None else s
            seen = (at > P - window) | (at < n_sink) if window else torch.ones(len(s), dtype=torch.bool)
            if not seen.any():
                continue
            k = rows64(new["k"], new["k_exp"], p[seen], h, r[seen])
            v = rows64(new["v"], new["v_exp"], p[seen], h, r[seen])
            qq = q[b, h * G:(h + 1) * G].double()
            every = torch.ones((G, len(k)), dtype=torch.bool)
            o, pr = attend64(qq, k, v, every)
            out[b, h * G:(h + 1) * G] = o
            tol[b, h * G:(h + 1) * G] = bound(qq, k, v, every, o, pr, out_dtype, False)
            mag = (qq.abs() @ k.abs().T / math.sqrt(d)).amax()
            rel = 2 * (mag * (d + 3) * 2.0 ** -24 + mag * 2.0 ** -22 + 2.0 ** -22 + len(k) * 2.0 ** -24)
            add[p[seen], h, r[seen]] = pr.sum(0)
            # the sum over the group and the addition to the score: G + 1 roundings
            old = new["score"][p[seen], h, r[seen]].double() if t["score"] is not None else 0.0
            add_tol[p[seen], h, r[seen]] = pr.sum(0) * rel + (G + 1) * 2.0 ** -24 * (pr.sum(0) + old) + 1e-38
    return out, tol, new, add, add_tol
