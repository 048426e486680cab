"""Performance cases of the paged key-value cache's operators.

One simulated step of a serving schedule stands for three calls on the cache
whose size the budget M counts in slots: ``append`` rotates a batch's new
queries and keys and writes keys and values into their pages, ``attend`` is
the attention of the new tokens over the pages (adding every slot's attention
weight to a running sum if asked to), ``evict`` shrinks sequences to a number
of slots by that sum.  Pools have the budgets of ``workloads.py`` (512, 65,536
and 262,144 slots) or what a sequence of the serving context needs; prompts
and answers have its lengths.

Fields of a case:
  op          ``append``, ``attend`` or ``evict``
  heads, kv_heads, dim, page, dtype   query and key heads, head size, slots of
              a page, type of everything but the 32-bit statistics
  seqs, ctx_lo, ctx_hi   sequences and the tokens that each holds already
  chunks, new_lo, new_hi   how many of them bring a chunk of new tokens, and of
              which length; the others bring one token (append, attend)
  slots       size of the pool
  rot, layout rotated part of the head, pairs ``half`` or ``interleaved`` (append)
  causal, window, weight   mask, and whether weights are summed (attend)
  budget, recent, first, aged   slots to keep, the newest and the first tokens
              that always stay, whether the cache was shrunk before (evict)
  shape       number from which ragged lengths are drawn: they belong to the
              case, another seed draws other values

``own = False``: plain torch in 32 bits.  ``own = True``: the package's kernels.
"""

import math
import random

import torch

own = False

#: Positions that the table of sines covers: the serving context.
POSITIONS = 65536


def _append(name, seqs, ctx, slots, heads=32, kv_heads=8, dim=128, page=16, dtype="bfloat16", rot=128,
            layout="half", chunks=0, new=(1, 1), shape=1):
    return {"name": name, "op": "append", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "slots": slots,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "rot": rot,
            "layout": layout, "chunks": chunks, "new_lo": new[0], "new_hi": new[1], "shape": shape}


def _attend(name, seqs, ctx, slots, heads=32, kv_heads=8, dim=128, page=16, dtype="bfloat16", causal=True,
            window=0, weight=False, chunks=0, new=(1, 1), shape=1):
    return {"name": name, "op": "attend", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "slots": slots,
            "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "causal": causal,
            "window": window, "weight": weight, "chunks": chunks, "new_lo": new[0], "new_hi": new[1],
            "shape": shape}


def _evict(name, seqs, ctx, slots, budget, recent, first=4, aged=False, kv_heads=8, dim=128, page=16,
           dtype="bfloat16", shape=1):
    return {"name": name, "op": "evict", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "slots": slots,
            "budget": budget, "recent": recent, "first": first, "aged": aged, "kv_heads": kv_heads, "dim": dim,
            "page": page, "dtype": dtype, "shape": shape}


def listed():
    return [
        # one request alone in the offline burst's pool: one layer's append, where the launch is the cost
        _append("append-one", 1, (31, 31), 512),
        # a decode step of the online workload: every running request appends its token
        _append("append-step", 203, (1, 600), 65536),
        # prompts admitted together: a chunk of each, interleaved pairs in half of the head
        _append("append-prompts", 9, (0, 700), 65536, dtype="float16", rot=64, layout="interleaved", chunks=9,
                new=(500, 4096)),
        # one request alone, its 64th token or so: latency
        _attend("attend-one", 1, (62, 62), 512),
        # a decode step of the online workload, ragged lengths
        _attend("attend-step", 127, (1, 900), 65536),
        # a decode step of the heavy-traffic workload, in which the cache keeps its weights for eviction
        _attend("attend-step-weight", 256, (64, 1850), 262144, weight=True),
        # one request at the end of the serving context, seven query heads to a key head
        _attend("attend-long", 1, (65534, 65534), 65552, heads=28, kv_heads=4, dtype="float16"),
        # a long prompt taken in pieces: a chunk of 2,048 behind 12,001 tokens, with weights
        _attend("attend-chunk-weight", 1, (12001, 12001), 65536, weight=True, chunks=1, new=(2048, 2048)),
        # prompts admitted together, nothing cached: the products bound it
        _attend("attend-prompts", 6, (0, 0), 65536, chunks=6, new=(700, 4096)),
        # one admitted prompt among running requests, small heads, one key head to each query head
        _attend("attend-mixed", 48, (1, 1500), 65536, heads=16, kv_heads=16, dim=64, chunks=1, new=(515, 515)),
        # every prompt of the heavy-traffic pool is shrunk after it was read
        _evict("evict-prompts", 64, (1025, 4096), 262144, 1024, 32),
        # the same requests some steps later: a few slots over the budget each
        _evict("evict-step", 48, (1056, 1056), 65536, 1024, 32, aged=True),
    ]


def _heads(rng):
    return rng.choice(((32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (8, 1, 128), (16, 2, 256), (12, 4, 64)))


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        heads, kv_heads, dim = _heads(rng)
        more = {"heads": heads, "kv_heads": kv_heads, "dim": dim, "page": rng.choice((1, 16, 16, 32, 64, 256)),
                "dtype": rng.choice(("bfloat16", "bfloat16", "float16")), "shape": rng.randrange(1 << 20)}
        op = rng.choice(("append", "attend", "attend", "attend", "evict"))
        seqs = size(1, 256)
        if op == "evict":
            del more["heads"]
            budget = size(64, 4096)
            aged = rng.random() < 0.5
            over = size(1, 64) if aged else size(16, 8192)
            recent = rng.randint(1, budget // 2)
            case = _evict(None, seqs, (budget + over, budget + over) if aged else (budget // 2, budget + over), 0,
                          budget, recent, first=rng.choice((0, 1, 4)), aged=aged, **more)
        else:
            chunked = rng.random() < 0.5
            if chunked:
                seqs = size(1, 48)
            hi = size(16, 16384)
            chunks = rng.randint(1, min(seqs, 8)) if chunked else 0
            new = (1, 1)
            if chunked:
                top = size(2, 4096)
                new = (max(1, top // 3), top)
            span = (rng.choice((0, hi // 4, hi)), hi)
            if op == "append":
                rot = rng.choice((dim, dim, dim // 2))
                case = _append(None, seqs, span, 0, rot=rot, layout=rng.choice(("half", "interleaved")),
                               chunks=chunks, new=new, **more)
            else:
                case = _attend(None, seqs, span, 0, causal=rng.random() < 0.8,
                               window=rng.choice((0, 0, 0, size(16, 4096))), weight=rng.random() < 0.4,
                               chunks=chunks, new=new, **more)
        del case["name"]
        case["slots"] = _needed(case) + case["page"] * rng.randint(0, 64)
        new, length = _lengths(case)
        slots = len(new) * max(length) * case["kv_heads"]
        if case["slots"] * case["kv_heads"] * dim > 1 << 28 or slots * dim > 1 << 29:
            continue        # more cache than the heavy-traffic workload's
        if op == "attend" and (slots * max(new) * heads // kv_heads > 1 << 31 or work(case)["flops"] > 2e11):
            continue        # more products than the prompts'
        return case


def _lengths(case):
    """(new tokens, length with them) of each sequence: the case's alone."""
    r = random.Random(case["shape"])
    length = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    if case["op"] == "evict":
        return [1] * len(length), length
    new = [r.randint(case["new_lo"], case["new_hi"]) if i < case["chunks"] else 1 for i in range(case["seqs"])]
    return new, [a + b for a, b in zip(length, new)]


def _needed(case):
    return sum(-(-x // case["page"]) for x in _lengths(case)[1]) * case["page"]


def work(case):
    new, length = _lengths(case)
    item, D, hk = 2, case["dim"], case["kv_heads"]
    pages = sum(-(-x // case["page"]) for x in length)
    if case["op"] == "evict":
        slots = moved = 0
        for n in length:
            over = n - case["budget"]
            if over <= 0:
                continue
            slots += n
            if over <= case["recent"]:
                moved += over
            else:           # the newest all move; of the others the weights decide, alike over the slots
                free = n - case["recent"] - case["first"]
                moved += case["recent"] + (over - case["recent"]) * (case["budget"] - case["recent"] - case["first"]) // free
        return {"bytes": hk * (8 * slots + moved * (8 + 4 * D * item)) + 4 * pages, "flops": 0}
    tokens, h = sum(new), case["heads"]
    if case["op"] == "append":
        return {"bytes": tokens * ((2 * h + 4 * hk) * D * item + 4 * case["rot"] + 4 + 8 * hk) + 4 * pages,
                "flops": 3 * tokens * (h + hk) * case["rot"]}
    pairs = seen = 0
    for n, m in zip(new, length):
        width = case["window"] or m
        if case["causal"]:
            pairs += sum(min(m - n + t + 1, width) for t in range(n))
            seen += min(m, width + n - 1)
        else:
            pairs += n * m
            seen += m
    return {"bytes": tokens * h * (2 * D * item + 4) + seen * hk * (2 * D * item + (8 if case["weight"] else 0)) + 4 * pages,
            "flops": 4 * D * h * pairs}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(22327 * 1000003 + int(seed))
    dev = dict(device="cuda", generator=g)
    ints = dict(device="cuda", dtype=torch.int32)
    dtype, D, hk, page = getattr(torch, case["dtype"]), case["dim"], case["kv_heads"], case["page"]
    new, length = _lengths(case)
    seqs, pool = case["seqs"], case["slots"] // page
    # pages in the order in which a pool that has been in use hands them out
    held = torch.tensor([-(-x // page) for x in length], device="cuda")
    wide = int(held.max())
    free = torch.randperm(pool, **dev)
    start = torch.cumsum(held, 0) - held
    at = torch.arange(wide, device="cuda")
    table = torch.where(at < held[:, None], free[(start[:, None] + at).clamp_(max=pool - 1)], 0).int()
    s = {"case": dict(case), "page_table": table, "kv_len": torch.tensor(length, **ints),
         "k": torch.randn((pool, hk, page, D), dtype=dtype, **dev),
         "v": torch.randn((pool, hk, page, D), dtype=dtype, **dev)}
    if case["op"] == "evict":
        L, budget = wide * page, case["budget"]
        slot = torch.arange(L, device="cuda")
        # sums of softmax weights spread over orders of magnitude; some underflowed to zero
        w = torch.exp(2 * torch.randn((seqs, hk, L), **dev))
        w = torch.where(torch.rand((seqs, hk, L), **dev) < 0.05, 0.0, w)
        pos = slot.expand(seqs, hk, L)
        after = s["kv_len"]
        if case["aged"]:
            # below the budget whatever an earlier eviction left, in its order; above it the tokens since then
            perm = torch.argsort(torch.rand((seqs, hk, budget), **dev), -1)
            after = s["kv_len"] + 1000
            newest = (after - s["kv_len"])[:, None, None] + slot
            old = torch.where(perm >= budget - 64, perm + 1000, perm)
            pos = newest.expand(seqs, hk, L).clone()
            pos[:, :, :budget] = old
        s["weight"], s["position"] = (torch.zeros((pool, hk, page), dtype=t, device="cuda")
                                      for t in (torch.float32, torch.int32))
        b, j = torch.nonzero(slot < s["kv_len"][:, None], as_tuple=True)
        pg = table.long()[b, j // page]
        s["weight"].transpose(1, 2)[pg, j % page] = w.transpose(1, 2)[b, j]
        s["position"].transpose(1, 2)[pg, j % page] = pos.int().transpose(1, 2)[b, j]
        s["next_position"] = after.int()
        return s
    tokens = sum(new)
    s["q_offsets"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
    s["max_q"] = max(new)
    H = case["heads"]
    if case["op"] == "append":
        # one projection's output: queries, keys and values of a token side by side
        qkv = torch.randn((tokens, H + 2 * hk, D), dtype=dtype, **dev)
        s["q"], s["k_new"], s["v_new"] = qkv[:, :H], qkv[:, H:H + hk], qkv[:, H + hk:]
        owner = torch.repeat_interleave(torch.arange(seqs, device="cuda"), torch.tensor(new, device="cuda"))
        t = torch.arange(tokens, device="cuda") - s["q_offsets"].long()[owner]
        s["positions"] = ((s["kv_len"] - torch.tensor(new, **ints))[owner] + t).int()
        rot = case["rot"]
        freq = 500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot) / 4
        angle = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * freq
        s["rope"] = torch.cat((angle.cos(), angle.sin()), 1).float()
        s["weight"] = torch.rand((pool, hk, page), **dev)
        s["position"] = torch.full((pool, hk, page), -1, **ints)
    else:
        s["q"] = torch.randn((tokens, H, D), dtype=dtype, **dev) * 1.5
        if case["weight"]:
            s["weight"] = torch.rand((pool, hk, page), **dev)
    return s


def run(state):
    return {"append": _run_append, "attend": _run_attend, "evict": _run_evict}[state["case"]["op"]](state)


def _package():
    from paper_2606_22327_amd import kvcache
    return kvcache


# -- append ------------------------------------------------------------------

def _rotate(x, cos, sin, layout):
    """x [T, heads, D] in 32 bits: its first 2 * cos.shape[1] dimensions turned."""
    r = 2 * cos.shape[1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if layout == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    c, s = cos[:, None], sin[:, None]
    y, z = a * c - b * s, b * c + a * s
    turned = torch.stack((y, z), -1).flatten(-2) if layout == "interleaved" else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _new_slots(s):
    """Page and row of every new token."""
    n = (s["q_offsets"][1:] - s["q_offsets"][:-1]).long()
    owner = torch.repeat_interleave(torch.arange(n.numel(), device=n.device), n)
    t = torch.arange(owner.numel(), device=n.device) - s["q_offsets"].long()[owner]
    slot = (s["kv_len"].long() - n)[owner] + t
    page = s["case"]["page"]
    return s["page_table"].long()[owner, slot // page], slot % page


def _run_append(s):
    case = s["case"]
    if own:
        C = _package()
        q = C.append(s["q"], s["k_new"], s["v_new"], s["positions"], s["rope"],
                     C.Batch(s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"]),
                     C.Cache(s["k"], s["v"], s["weight"], s["position"]), layout=case["layout"])
    else:
        row = s["rope"][s["positions"].long()]
        cos, sin = row[:, :case["rot"] // 2], row[:, case["rot"] // 2:]
        q = _rotate(s["q"].float(), cos, sin, case["layout"]).to(s["q"].dtype)
        page, off = _new_slots(s)
        s["k"].transpose(1, 2)[page, off] = _rotate(s["k_new"].float(), cos, sin, case["layout"]).to(s["k"].dtype)
        s["v"].transpose(1, 2)[page, off] = s["v_new"]
        s["weight"].transpose(1, 2)[page, off] = 0.0
        s["position"].transpose(1, 2)[page, off] = s["positions"][:, None]
    return {"q": q, "k": s["k"], "v": s["v"], "weight": s["weight"], "position": s["position"]}


# -- attend ------------------------------------------------------------------

def _run_attend(s):
    case = s["case"]
    weight = s["weight"].clone() if case["weight"] else None
    if own:
        C = _package()
        out, lse = C.attend(s["q"], C.Batch(s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"]),
                            C.Cache(s["k"], s["v"], weight), causal=case["causal"], window=case["window"],
                            add_weight=case["weight"])
    else:
        out, lse = _plain_attend(s, case, weight)
    return {"out": out, "lse": lse} if weight is None else {"out": out, "lse": lse, "weight": weight}


def _plain_attend(s, case, weight):
    table, n_max, D, hk = s["page_table"].long(), s["max_q"], case["dim"], case["kv_heads"]
    B, L, G, page = table.shape[0], table.shape[1] * case["page"], case["heads"] // hk, case["page"]
    first, length = s["q_offsets"][:-1].long(), s["kv_len"].long()
    n = s["q_offsets"][1:].long() - first
    t, slot = torch.arange(n_max, device=table.device), torch.arange(L, device=table.device)
    real = t < n[:, None]
    q = s["q"][(first[:, None] + t).clamp_(max=s["q"].shape[0] - 1)].float()
    q = q.view(B, n_max, hk, G, D).transpose(1, 2).reshape(B, hk, n_max * G, D)
    k = s["k"][table].transpose(1, 2).reshape(B, hk, L, D).float()
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, hk, n_max, G, L)
    del q, k
    last = ((length - n)[:, None] + t if case["causal"] else (length - 1)[:, None].expand(B, n_max))[:, :, None]
    hidden = (slot > last) | ~real[:, :, None] | (slot >= length[:, None, None])
    if case["window"]:
        hidden |= slot <= (length - n)[:, None, None] + t[:, None] - case["window"]
    score.masked_fill_(hidden[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1).transpose(1, 2).reshape(B, n_max, -1)[real]
    p /= torch.where(total > 0, total, 1.0)
    v = s["v"][table].transpose(1, 2).reshape(B, hk, L, D).float()
    out = torch.matmul(p.view(B, hk, n_max * G, L), v)
    out = out.view(B, hk, n_max, G, D).transpose(1, 2).reshape(B, n_max, hk * G, D)[real].to(s["q"].dtype)
    if weight is not None:
        b, j = torch.nonzero(slot < length[:, None], as_tuple=True)
        weight.transpose(1, 2)[table[b, j // page], j % page] += p.sum((2, 3)).transpose(1, 2)[b, j]
    return out, lse


# -- evict -------------------------------------------------------------------

def _run_evict(s):
    case = s["case"]
    weight, position = s["weight"].clone(), s["position"].clone()
    if own:
        C = _package()
        length = C.evict(C.Batch(None, s["kv_len"], s["page_table"], 0), C.Cache(s["k"], s["v"], weight, position),
                         case["budget"], recent=case["recent"], first=case["first"],
                         next_position=s["next_position"])
    else:
        length = _plain_evict(s, case, weight, position)
    return {"length": length, "k": s["k"], "v": s["v"], "weight": weight, "position": position}


def _plain_evict(s, case, weight, position):
    table, page, hk, budget = s["page_table"].long(), case["page"], case["kv_heads"], case["budget"]
    B, L = table.shape[0], table.shape[1] * page
    slot = torch.arange(L, device=table.device)
    length = s["kv_len"].long()[:, None, None]
    w = weight[table].transpose(1, 2).reshape(B, hk, L)
    pos = position[table].transpose(1, 2).reshape(B, hk, L)
    after = s["next_position"].long()[:, None, None]
    key = torch.where((pos < case["first"]) | (pos >= after - case["recent"]), math.inf, w)
    key = torch.where(slot < length, key, -math.inf)
    order = torch.argsort(key, dim=-1, descending=True, stable=True)
    kept = torch.zeros((B, hk, L), dtype=torch.bool, device=table.device).scatter_(2, order[:, :, :budget], True)
    over = length > budget
    hb, hh, hj = torch.nonzero(~kept & over & (slot < budget), as_tuple=True)
    mb, mh, mj = torch.nonzero(kept & over & (slot >= budget), as_tuple=True)
    to, at = (table[hb, hj // page], hh, hj % page), (table[mb, mj // page], mh, mj % page)
    for x in (s["k"], s["v"], weight, position):
        x[to] = x[at]
    return s["kv_len"].clamp(max=budget)


# -- the definitions in 64 bits, sequence by sequence --------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict}[case["op"]](s, case)


def _exact_append(s, case):
    half, D = case["rot"] // 2, case["dim"]
    angle = torch.atan2(s["rope"][:, half:].double(), s["rope"][:, :half].double())
    size = torch.hypot(s["rope"][:, half:].double(), s["rope"][:, :half].double())
    unit = torch.polar(size, angle)[s["positions"].long()][:, None]

    def turn(x):
        x = x.double()
        y = x.clone()
        i = torch.arange(half, device=x.device)
        a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + half)
        z = torch.complex(x[..., a], x[..., b]) * unit
        y[..., a], y[..., b] = z.real, z.imag
        return y

    k, v = s["k"].double(), s["v"].double()
    weight, position = s["weight"].double(), s["position"].clone()
    kr, at, offs, lens = turn(s["k_new"]), 0, s["q_offsets"].tolist(), s["kv_len"].tolist()
    for i, length in enumerate(lens):
        n = offs[i + 1] - offs[i]
        slot = torch.arange(length - n, length, device=k.device)
        pg, row = s["page_table"][i].long()[slot // case["page"]], slot % case["page"]
        for h in range(case["kv_heads"]):
            k[pg, h, row], v[pg, h, row] = kr[at:at + n, h], s["v_new"][at:at + n, h].double()
            weight[pg, h, row], position[pg, h, row] = 0.0, s["positions"][at:at + n]
        at += n
    return {"q": turn(s["q"]), "k": k, "v": v, "weight": weight, "position": position}


def _exact_attend(s, case):
    H, hk, page = case["heads"], case["kv_heads"], case["page"]
    q, offs = s["q"].double(), s["q_offsets"].tolist()
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=q.device)
    weight = s["weight"].double() if case["weight"] else None
    for i, length in enumerate(s["kv_len"].tolist()):
        a, b = offs[i], offs[i + 1]
        slot = torch.arange(length, device=q.device)
        row = length - (b - a) + torch.arange(b - a, device=q.device)[:, None]
        seen = (slot <= row) if case["causal"] else (slot >= 0).expand(b - a, length)
        if case["window"]:
            seen = seen & (slot > row - case["window"])
        pg, off = s["page_table"][i].long()[slot // page], slot % page
        for h in range(hk):
            g = slice(h * (H // hk), (h + 1) * (H // hk))
            sc = torch.einsum("thd,jd->htj", q[a:b, g], s["k"][pg, h, off].double()) / math.sqrt(case["dim"])
            sc = sc.masked_fill(~seen, -math.inf)
            total = torch.logsumexp(sc, -1, keepdim=True)
            p = torch.exp(sc - total)
            out[a:b, g] = torch.einsum("htj,jd->thd", p, s["v"][pg, h, off].double())
            lse[a:b, g] = total.squeeze(-1).T
            if weight is not None:
                weight[pg, h, off] += p.sum((0, 1))
    return {"out": out, "lse": lse} if weight is None else {"out": out, "lse": lse, "weight": weight}


def _exact_evict(s, case):
    page, budget = case["page"], case["budget"]
    k, v, weight, position = s["k"].double(), s["v"].double(), s["weight"].double(), s["position"].clone()
    for i, length in enumerate(s["kv_len"].tolist()):
        if length <= budget:
            continue
        slot = torch.arange(length, device=k.device)
        pg, off = s["page_table"][i].long()[slot // page], slot % page
        pos, w = position[pg, :, off], weight[pg, :, off]                    # [length, heads]
        w[(pos < case["first"]) | (pos >= int(s["next_position"][i]) - case["recent"])] = math.inf
        # the budget-th largest, and as many of its equals as there is room for
        edge = torch.sort(w, 0).values[length - budget]
        room = budget - (w > edge).sum(0)
        equal = w == edge
        keep = (w > edge) | (equal & (equal.cumsum(0) <= room))
        for h in range(case["kv_heads"]):
            to, at = slot[:budget][~keep[:budget, h]], slot[budget:][keep[budget:, h]]
            for x in (k, v, weight, position):
                x[pg[to], h, off[to]] = x[pg[at], h, off[at]]
    return {"length": s["kv_len"].clamp(max=budget), "k": k, "v": v, "weight": weight, "position": position}
