"""Plain 64-bit forms of the paged cache's operators, on the CPU: sequence by
sequence, written from the definitions in include/svfkv.h."""

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a step of a number just above a power of two, relative


def slots_of(table, i, length, page, num_pages):
    """(page, row) of each slot of sequence i; page -1 where there is none."""
    length = max(0, min(int(length), table.shape[1] * page))
    j = torch.arange(length)
    pg = table[i].long()[j // page] if length else torch.empty(0, dtype=torch.long)
    return torch.where((pg < 0) | (pg >= num_pages), -1, pg), j % page


def rotate(x, angle_cos, angle_sin, layout):
    """x [T, heads, D] in 64 bits; cosines and sines [T, rot / 2]."""
    half = angle_cos.shape[1]
    y = x.clone()
    for i in range(half):
        a, b = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = angle_cos[:, i, None], angle_sin[:, i, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def attend(q, k, v, offsets, kv_len, table, causal, window, scale):
    """(out, lse, weight, tol): all in 64 bits; ``weight`` is what is added; ``tol`` holds what
    the tolerances are derived from: sum_j p|v| per output and the largest |scale| * sum|q||k| per row."""
    q = q.double()
    T, H, D = q.shape
    pages, hk, page = k.shape[:3]
    G = H // hk
    out = torch.zeros_like(q)
    absv = torch.zeros_like(q)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64)
    big = torch.zeros((T, H), dtype=torch.float64)
    weight = torch.zeros((pages, hk, page), dtype=torch.float64)
    for i in range(len(kv_len)):
        a, b = int(offsets[i]), int(offsets[i + 1])
        pg, row = slots_of(table, i, kv_len[i], page, pages)
        n, m = b - a, len(pg)
        if n == 0 or m == 0:
            continue
        r = m - n + torch.arange(n)[:, None]
        j = torch.arange(m)
        seen = (pg >= 0) & (j <= r if causal else j >= 0) & (j > r - window if window else j >= 0)
        seen, there = seen.expand(n, m), pg >= 0
        for h in range(hk):
            kk, vv = k[pg.clamp(min=0), h, row].double(), v[pg.clamp(min=0), h, row].double()
            kk = torch.where(there[:, None], kk, 0.0)
            vv = torch.where(there[:, None], vv, 0.0)
            for g in range(h * G, (h + 1) * G):
                s = torch.where(seen, scale * (q[a:b, g] @ kk.T), -math.inf)
                top = s.amax(1, keepdim=True)
                e = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
                total = e.sum(1, keepdim=True)
                p = torch.where(total != 0, e / total, 0.0)
                for x in range(n):          # only what a row sees enters its sums
                    w = seen[x]
                    out[a + x, g] = p[x, w] @ vv[w]
                    absv[a + x, g] = p[x, w] @ vv[w].abs()
                    big[a + x, g] = (abs(scale) * (kk[w].abs() @ q[a + x, g].abs())).max() if w.any() else 0.0
                lse[a:b, g] = (top + total.log()).squeeze(1)
                ps = p.sum(0)
                weight[pg[there], h, row[there]] += ps[there]
    return out, lse, weight, {"absv": absv, "big": big}


def out_tolerance(dtype, D, out, tol, slots):
    """|error| of an output: the probabilities and the output are rounded to the type (UNIT each, of
    sum p|v| and of |out|); a score is a sum of D products in 32 bits (D steps of 2^-23 of sum|q||k|,
    which is a relative error of the probability, once in it and once in their sum), exponential and sums a
    few steps more; 16-bit floats below 2^-14 have an absolute step, with the probabilities scaled by 2^14."""
    rel = 2 * (D * 2.0 ** -23 * tol["big"] + 2.0 ** -18)
    e = UNIT[dtype] * (out.abs() + tol["absv"]) + rel[..., None] * tol["absv"]
    if dtype == torch.float16:
        e = e + 2.0 ** -25 * out.abs().clamp(min=2.0 ** -14) + slots * 2.0 ** -39 * 8
    return e * 1.01 + 1e-30


def lse_tolerance(D, lse, tol):
    return D * 2.0 ** -23 * tol["big"] + 2.0 ** -18 + 2.0 ** -21 * lse.abs()


def weight_tolerance(D, base, weight, tol, rows):
    rel = 2 * (D * 2.0 ** -23 * float(tol["big"].max()) + 2.0 ** -18) + rows * 2.0 ** -23
    return rel * weight + 2.0 ** -23 * (base.abs() + weight) + 1e-30


def evict(k, v, weight, position, kv_len, table, budget, recent, first, after):
    """The cache after eviction and the new lengths (copies)."""
    k, v, weight, position = k.clone(), v.clone(), weight.clone(), position.clone()
    pages, hk, page = k.shape[:3]
    new = []
    for i in range(len(kv_len)):
        pg, row = slots_of(table, i, kv_len[i], page, pages)
        m = len(pg)
        new.append(min(m, budget))
        if m <= budget:
            continue
        for h in range(hk):
            rank = []
            for j in range(m):
                if pg[j] < 0:
                    rank.append((2, 0.0, j))
                    continue
                w, pos = float(weight[pg[j], h, row[j]]), int(position[pg[j], h, row[j]])
                if pos < first or pos >= int(after[i]) - recent:
                    rank.append((0, 0.0, j))
                elif w != w:
                    rank.append((2, 0.0, j))
                else:
                    rank.append((1, -w, j))
            kept = sorted(x[2] for x in sorted(rank)[:budget])
            movers = [j for j in kept if j >= budget]
            stay = set(kept)
            holes = [j for j in range(budget) if j not in stay]
            assert len(holes) == len(movers)
            for to, at in zip(holes, movers):
                if pg[to] < 0 or pg[at] < 0:
                    continue
                for x in (k, v, weight, position):
                    x[pg[to], h, row[to]] = x[pg[at], h, row[at]]
    return k, v, weight, position, torch.tensor(new, dtype=torch.int32)
