"""Performance cases of the calls that serve images, endless texts and scored answers.

What a step of a request does beyond the cases of ``operators.py``:

``append`` with ``axes``   tokens of images and videos have positions with several axes
              (time, height, width): every pair of a head turns by one of them
``attend`` with ``first``   a window in which the first tokens stay visible, so that a text
              may go on past any budget; the pages between were given back
``logprobs.score``   what the step's answers are worth: log probabilities of given tokens,
              their ranks, entropies and the best alternatives, from logits

Pools, prompts and answers have the lengths of ``workloads.py`` (budgets of 512, 65,536
and 262,144 slots) and the serving context's.

Fields of a case:
  op          ``append``, ``attend`` or ``score``
  heads, kv_heads, dim, page, dtype   query and key heads, head size, slots of
              a page, type of everything but the 32-bit statistics (``score``: of the logits)
  seqs, ctx_lo, ctx_hi   sequences and the tokens that each holds already
  chunks, new_lo, new_hi   how many of them bring a chunk of new tokens, and of
              which length; the others bring one token
  layout      pairs ``half`` or ``interleaved``; p0, p1, p2: pairs of each axis; cyclic: whether
              the axes take turns, not blocks of pairs (append)
  grid_h, grid_w   tokens of an image; images and runs of text follow each other (append)
  window, first, weight   mask, and whether weights are summed (attend)
  freed       whether pages that no token will see again are given back (attend)
  rows, vocab, stride, top, scale   logits and the distance of their rows, alternatives, inverse temperature
  banned      share of the vocabulary that a grammar rules out (logits of -inf) (score)
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


def _append(name, seqs, ctx, pairs, heads=32, kv_heads=8, dim=128, page=16, dtype="bfloat16", layout="half",
            cyclic=False, grid=(32, 32), chunks=0, new=(1, 1), shape=1):
    return {"name": name, "op": "append", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype, "layout": layout, "p0": pairs[0],
            "p1": pairs[1], "p2": pairs[2], "cyclic": cyclic, "grid_h": grid[0], "grid_w": grid[1],
            "chunks": chunks, "new_lo": new[0], "new_hi": new[1], "shape": shape}


def _attend(name, seqs, ctx, window, first, heads=32, kv_heads=8, dim=128, page=16, dtype="bfloat16", weight=False,
            freed=True, chunks=0, new=(1, 1), shape=1):
    return {"name": name, "op": "attend", "seqs": seqs, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "window": window,
            "first": first, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype,
            "weight": weight, "freed": freed, "chunks": chunks, "new_lo": new[0], "new_hi": new[1], "shape": shape}


def _score(name, rows, vocab, top, dtype="bfloat16", stride=0, scale=1.0, banned=0.0):
    return {"name": name, "op": "score", "rows": rows, "vocab": vocab, "stride": stride or vocab, "top": top,
            "dtype": dtype, "scale": scale, "banned": banned}


def listed():
    return [
        # a decode step of the online workload whose requests hold images: every running request appends its token
        _append("axes-step", 203, (1, 600), (16, 24, 24)),
        # prompts of texts and images of 32 x 32 tokens admitted together
        _append("axes-images", 9, (0, 700), (16, 24, 24), chunks=9, new=(500, 4096)),
        # one long video, 24 x 42 tokens a frame, the axes taking turns over three quarters of the head
        _append("axes-video", 1, (0, 0), (16, 16, 16), dtype="float16", layout="interleaved", cyclic=True,
                grid=(24, 42), chunks=1, new=(32001, 32001)),
        # one request alone, some tokens past its window: latency
        _attend("first-one", 1, (99, 99), 64, 4),
        # a decode step of the heavy-traffic workload in windows, with weights kept
        _attend("first-step-weight", 256, (64, 4000), 1024, 4, weight=True),
        # one request at the end of the serving context, seven query heads to a key head, all pages still held
        _attend("first-long", 1, (65534, 65534), 16384, 64, heads=28, kv_heads=4, dtype="float16", freed=False),
        # a long prompt taken in pieces: a chunk of 2,048 behind 12,001 tokens, with weights
        _attend("first-chunk-weight", 1, (12001, 12001), 4096, 16, weight=True, chunks=1, new=(2048, 2048)),
        # prompts admitted together, nothing cached, small heads, one key head to each query head
        _attend("first-prompts", 6, (0, 0), 512, 128, heads=16, kv_heads=16, dim=64, chunks=6, new=(700, 4096)),
        # the answer of one request
        _score("score-one", 1, 32000, 5),
        # a decode step's answers under a grammar
        _score("score-step", 203, 128000, 20, banned=0.3),
        # the prompts admitted together, scored whole: the logits' buffer bounds it
        _score("score-prompts", 4001, 128000, 1),
        # a vocabulary of odd size in 32 bits, at a temperature of 0.7, out of a padded buffer
        _score("score-odd", 517, 50001, 8, dtype="float32", stride=50047, scale=1 / 0.7),
    ]


def _heads(rng):
    return rng.choice(((32, 8, 128), (32, 8, 128), (28, 4, 128), (16, 16, 64), (8, 1, 128), (16, 2, 256), (12, 4, 64)))


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(("append", "attend", "attend", "score"))
        if op == "score":
            rows, vocab = size(1, 4096), size(1000, 160000)
            dtype = rng.choice(("bfloat16", "bfloat16", "float16", "float32"))
            case = _score(None, rows, vocab, rng.choice((0, 1, 5, 20, 64)), dtype, vocab + rng.choice((0, 0, rng.randint(1, 128))),
                          rng.choice((1.0, 1.0, round(rng.uniform(0.5, 3.0), 3))), rng.choice((0.0, 0.0, 0.5)))
            if rows * vocab * (4 if dtype == "float32" else 2) > 1 << 30:
                continue        # more than the prompts' logits
            del case["name"]
            return case
        heads, kv_heads, dim = _heads(rng)
        more = {"heads": heads, "kv_heads": kv_heads, "dim": dim, "page": rng.choice((1, 16, 16, 32, 64, 256)),
                "dtype": rng.choice(("bfloat16", "bfloat16", "float16")), "shape": rng.randrange(1 << 20)}
        chunked = rng.random() < 0.5
        seqs = size(1, 48 if chunked else 256)
        chunks = rng.randint(1, min(seqs, 8)) if chunked else 0
        new = (1, 1)
        if chunked:
            most = size(2, 4096)
            new = (max(1, most // 3), most)
        hi = size(16, 16384)
        span = (rng.choice((0, hi // 4, hi)), hi)
        if op == "append":
            third = rng.randint(1, dim // 6)
            pairs = rng.choice(((dim // 2 - 2 * third, third, third), (third, third, third)))
            case = _append(None, seqs, span, pairs, layout=rng.choice(("half", "interleaved")),
                           cyclic=rng.random() < 0.5, grid=(size(4, 64), size(4, 64)), chunks=chunks, new=new, **more)
        else:
            case = _attend(None, seqs, span, size(16, 8192), rng.choice((1, 4, size(1, 256))),
                           weight=rng.random() < 0.4, freed=rng.random() < 0.6, chunks=chunks, new=new, **more)
        del case["name"]
        n, length = _lengths(case)
        slots = len(n) * max(length) * kv_heads
        w = work(case)
        if sum(length) * kv_heads * dim > 1 << 29 or slots * dim > 1 << 30 or w["bytes"] > 1.1e9:
            continue        # more cache than the heavy-traffic workload's step
        if op == "attend" and (slots * max(n) * heads // kv_heads > 1 << 31 or w["flops"] > 1.2e11):
            continue        # more products than the long prompt's chunk
        return case


def _lengths(case):
    """(new tokens, length with them) of each sequence: the case's alone."""
    r = random.Random(case["shape"])
    length = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["seqs"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) if i < case["chunks"] else 1 for i in range(case["seqs"])]
    return new, [a + b for a, b in zip(length, new)]


def work(case):
    if case["op"] == "score":
        rows, item = case["rows"], 4 if case["dtype"] == "float32" else 2
        # a difference, an exponential, and a sum of it and of it times the difference
        return {"bytes": rows * (case["vocab"] * item + 8 + 12 + 8 * case["top"]), "flops": 5 * rows * case["vocab"]}
    new, length = _lengths(case)
    item, D, h, hk = 2, case["dim"], case["heads"], case["kv_heads"]
    tokens, pages = sum(new), sum(-(-x // case["page"]) for x in length)
    if case["op"] == "append":
        rot = 2 * (case["p0"] + case["p1"] + case["p2"])
        return {"bytes": tokens * ((2 * h + 4 * hk) * D * item + 4 * rot + 16 + 8 * hk) + 4 * pages,
                "flops": 3 * tokens * (h + hk) * rot}
    pairs = seen = 0
    for n, m in zip(new, length):
        for r in range(m - n, m):
            pairs += min(r + 1, case["window"] + min(case["first"], max(0, r + 1 - case["window"])))
        seen += min(m, case["window"] + n - 1 + min(case["first"], max(0, m - n - case["window"] + 1)))
    return {"bytes": tokens * h * (2 * D * item + 4) + seen * hk * (2 * D * item + (8 if case["weight"] else 0)) + 4 * pages,
            "flops": 4 * D * h * pairs}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(22327 * 1000003 + int(seed))
    return (_prepare_score if case["op"] == "score" else _prepare_cache)(case, g)


def _prepare_score(case, g):
    dev = dict(device="cuda", generator=g)
    rows, vocab = case["rows"], case["vocab"]
    # some hundred likely tokens in a long tail, one of them far ahead in half of the rows
    x = torch.randn((rows, case["stride"]), dtype=getattr(torch, case["dtype"]), **dev).mul_(2.5)[:, :vocab]
    row = torch.arange(rows, device="cuda")
    ahead = torch.randint(vocab, (rows,), **dev)
    x[row, ahead] += 10.0 * torch.rand((rows,), **dev).round().to(x.dtype) + 6.0
    if case["banned"]:
        x.masked_fill_(torch.rand((vocab,), **dev) < case["banned"], -math.inf)
    # the likely token, or any other
    token = torch.where(torch.rand((rows,), **dev) < 0.7, ahead, torch.randint(vocab, (rows,), **dev))
    return {"case": dict(case), "logits": x, "token": token}


def _prepare_cache(case, g):
    dev = dict(device="cuda", generator=g)
    ints = dict(device="cuda", dtype=torch.int32)
    dtype, D, hk, page = getattr(torch, case["dtype"]), case["dim"], case["kv_heads"], case["page"]
    new, length = _lengths(case)
    seqs, tokens = case["seqs"], sum(new)
    n, m = torch.tensor(new, device="cuda"), torch.tensor(length, device="cuda")
    # pages in the order in which a pool that has been in use hands them out; -1 where one was given back
    at = torch.arange(max(-(-x // page) for x in length), device="cuda")
    there = at < ((m + page - 1) // page)[:, None]
    if case["op"] == "attend" and case["freed"]:
        oldest = (m - n - case["window"] + 1)[:, None]      # that the first new token sees
        there &= (at * page < case["first"]) | ((at + 1) * page > oldest)
    held = int(there.sum())
    pool = held + 16
    table = torch.full(there.shape, -1, **ints)
    table[there] = torch.randperm(pool, **dev)[:held].int()
    s = {"case": dict(case), "page_table": table, "kv_len": m.int(), "max_q": max(new),
         "q_offsets": torch.tensor([0] + new, device="cuda").cumsum(0).int(),
         "k": torch.randn((pool, hk, page, D), dtype=dtype, **dev),
         "v": torch.randn((pool, hk, page, D), dtype=dtype, **dev)}
    H = case["heads"]
    if case["op"] == "attend":
        s["q"] = torch.randn((tokens, H, D), dtype=dtype, **dev) * 1.5
        if case["weight"]:
            s["weight"] = torch.rand((pool, hk, page), **dev)
        return s
    # one projection's output: queries, keys and values of a token side by side
    qkv = torch.randn((tokens, H + 2 * hk, D), dtype=dtype, **dev)
    s["q"], s["k_new"], s["v_new"] = qkv[:, :H], qkv[:, H:H + hk], qkv[:, H + hk:]
    owner = torch.repeat_interleave(torch.arange(seqs, device="cuda"), n)
    token = (m - n)[owner] + torch.arange(tokens, device="cuda") - s["q_offsets"].long()[owner]
    # each image follows 100 tokens of text: time stands still in it, rows and columns count from there
    gh, gw = case["grid_h"], case["grid_w"]
    turn, i = token // (100 + gh * gw), token % (100 + gh * gw)
    start, inside = turn * (100 + max(gh, gw)) + i.clamp(max=100), (i - 100).clamp_(min=0)
    s["positions"] = torch.stack((start, start + inside // gw, start + inside % gw), 1).int()
    s["token"] = token.int()
    pairs = (case["p0"], case["p1"], case["p2"])
    half = sum(pairs)
    s["pairs"] = pairs
    # which axis a pair turns by: in blocks, or in turns until an axis has all of its pairs
    axis = [a for a in range(3) for _ in range(pairs[a])]
    if case["cyclic"]:
        axis = [a for i in range(max(pairs)) for a in range(3) if i < pairs[a]]
    s["axis"] = torch.tensor(axis, device="cuda")
    s["axes"] = bytes(axis)
    freq = 500000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = torch.arange(POSITIONS, device="cuda", dtype=torch.float64)[:, None] * freq
    s["rope"] = torch.cat((angle.cos(), angle.sin()), 1).float()
    s["weight"] = torch.rand((pool, hk, page), **dev)
    s["position"] = torch.full((pool, hk, page), -1, **ints)
    return s


def run(state):
    return {"append": _run_append, "attend": _run_attend, "score": _run_score}[state["case"]["op"]](state)


# -- append ------------------------------------------------------------------

def _rotate(x, cos, sin, layout):
    """x [T, heads, D] in 32 bits: its first 2 * cos.shape[1] dimensions turned."""
    r = 2 * cos.shape[1]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if layout == "interleaved" else (x[..., :r // 2], x[..., r // 2:r])
    c, s = cos[:, None], sin[:, None]
    y, z = a * c - b * s, b * c + a * s
    turned = torch.stack((y, z), -1).flatten(-2) if layout == "interleaved" else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., r:]), -1)


def _run_append(s):
    case = s["case"]
    if own:
        from paper_2606_22327_amd import kvcache as C
        q = C.append(s["q"], s["k_new"], s["v_new"], s["positions"], s["rope"],
                     C.Batch(s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"]),
                     C.Cache(s["k"], s["v"], s["weight"], s["position"]), layout=case["layout"], axes=s["axes"],
                     kept=s["token"])
    else:
        pair = torch.arange(s["axis"].numel(), device=s["axis"].device)
        at = s["positions"].long()[:, s["axis"]]
        cos, sin = s["rope"][at, pair], s["rope"][at, pair + pair.numel()]
        q = _rotate(s["q"].float(), cos, sin, case["layout"]).to(s["q"].dtype)
        n = (s["q_offsets"][1:] - s["q_offsets"][:-1]).long()
        owner = torch.repeat_interleave(torch.arange(n.numel(), device=n.device), n)
        slot = (s["kv_len"].long() - n)[owner] + torch.arange(owner.numel(), device=n.device) - s["q_offsets"].long()[owner]
        page, off = s["page_table"].long()[owner, slot // case["page"]], slot % case["page"]
        s["k"].transpose(1, 2)[page, off] = _rotate(s["k_new"].float(), cos, sin, case["layout"]).to(s["k"].dtype)
        s["v"].transpose(1, 2)[page, off] = s["v_new"]
        s["weight"].transpose(1, 2)[page, off] = 0.0
        s["position"].transpose(1, 2)[page, off] = s["token"][:, None]
    return {"q": q, "k": s["k"], "v": s["v"], "weight": s["weight"], "position": s["position"]}


# -- attend ------------------------------------------------------------------

def _run_attend(s):
    case = s["case"]
    weight = s["weight"].clone() if case["weight"] else None
    if own:
        from paper_2606_22327_amd import kvcache as C
        out, lse = C.attend(s["q"], C.Batch(s["q_offsets"], s["kv_len"], s["page_table"], s["max_q"]),
                            C.Cache(s["k"], s["v"], weight), window=case["window"], first=case["first"],
                            add_weight=case["weight"])
    else:
        out, lse = _plain_attend(s, case, weight)
    return {"out": out, "lse": lse} if weight is None else {"out": out, "lse": lse, "weight": weight}


def _plain_attend(s, case, weight):
    table, n_max, D, hk = s["page_table"].long(), s["max_q"], case["dim"], case["kv_heads"]
    B, L, G, page = table.shape[0], table.shape[1] * case["page"], case["heads"] // hk, case["page"]
    begin, length = s["q_offsets"][:-1].long(), s["kv_len"].long()
    n = s["q_offsets"][1:].long() - begin
    t, slot = torch.arange(n_max, device=table.device), torch.arange(L, device=table.device)
    real = t < n[:, None]
    held = (table >= 0).repeat_interleave(page, 1) & (slot < length[:, None])
    table = table.clamp(min=0)
    q = s["q"][(begin[:, None] + t).clamp_(max=s["q"].shape[0] - 1)].float()
    q = q.view(B, n_max, hk, G, D).transpose(1, 2).reshape(B, hk, n_max * G, D)
    k = s["k"][table].transpose(1, 2).reshape(B, hk, L, D).float()
    score = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(D ** -0.5).view(B, hk, n_max, G, L)
    del q, k
    row = ((length - n)[:, None] + t)[:, :, None]
    seen = (slot <= row) & ((slot > row - case["window"]) | (slot < case["first"])) & held[:, None] & real[:, :, None]
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
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
        b, j = torch.nonzero(held, as_tuple=True)
        weight.transpose(1, 2)[table[b, j // page], j % page] += p.sum((2, 3)).transpose(1, 2)[b, j]
    return out, lse


# -- score -------------------------------------------------------------------

def _run_score(s):
    case = s["case"]
    if own:
        from paper_2606_22327_amd import logprobs
        r = logprobs.score(s["logits"], s["token"], top=case["top"], scale=case["scale"])
        return {"logprob": r.logprob, "entropy": r.entropy, "rank": r.rank, "top_logprob": r.top_logprob,
                "top_index": r.top_index}
    x, token = s["logits"].float(), s["token"][:, None]
    index = torch.arange(case["vocab"], device=x.device)
    mine = x.gather(1, token)
    rank = ((x > mine) | ((x == mine) & (index < token))).sum(1).int()
    # the order of numbers as the order of whole numbers, the index behind it
    bits = (x + 0.0).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 4294967296 + (4294967295 - index)
    top_index = 4294967295 - (torch.topk(key, case["top"], dim=1).values & 0xFFFFFFFF)
    del key, bits
    most = x.amax(1, keepdim=True)
    x = (x - most).mul_(case["scale"])
    e = x.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    logprob = (x.gather(1, token) - log_total).squeeze(1)
    top_logprob = x.gather(1, top_index) - log_total
    mean = torch.where(e > 0, x, 0.0).mul_(e).sum(1, keepdim=True) / total
    return {"logprob": logprob, "entropy": (log_total - mean).squeeze(1), "rank": rank, "top_logprob": top_logprob,
            "top_index": top_index.int()}


# -- the definitions in 64 bits, sequence by sequence --------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "score": _exact_score}[case["op"]](s, case)


def _exact_append(s, case):
    half = sum(s["pairs"])
    k, v = s["k"].double(), s["v"].double()
    weight, position = s["weight"].double(), s["position"].clone()
    unit = torch.complex(s["rope"][:, :half].double(), s["rope"][:, half:].double())
    turn_by = torch.empty((s["positions"].shape[0], half), dtype=torch.complex128, device=k.device)
    given = list(s["pairs"])
    at = 0
    for p in range(half):           # the axis of pair p, counted out anew
        if case["cyclic"]:
            while given[at % 3] == 0:
                at += 1
            a = at % 3
            at += 1
        else:
            a = next(i for i in range(3) if given[i])
        given[a] -= 1
        turn_by[:, p] = unit[s["positions"][:, a].long(), p]

    def turn(x):
        x = x.double()
        y = x.clone()
        i = torch.arange(half, device=x.device)
        a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + half)
        z = torch.complex(x[..., a], x[..., b]) * turn_by[:, None]
        y[..., a], y[..., b] = z.real, z.imag
        return y

    kr, at, offs = turn(s["k_new"]), 0, s["q_offsets"].tolist()
    for i, length in enumerate(s["kv_len"].tolist()):
        n = offs[i + 1] - offs[i]
        slot = torch.arange(length - n, length, device=k.device)
        pg, row = s["page_table"][i].long()[slot // case["page"]], slot % case["page"]
        for h in range(case["kv_heads"]):
            k[pg, h, row], v[pg, h, row] = kr[at:at + n, h], s["v_new"][at:at + n, h].double()
            weight[pg, h, row], position[pg, h, row] = 0.0, slot.int()
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
        slot = slot[s["page_table"][i].long()[slot // page] >= 0]       # what is still held
        own_slot = length - (b - a) + torch.arange(b - a, device=q.device)[:, None]
        far = own_slot - slot
        seen = (far >= 0) & ((far < case["window"]) | (slot < case["first"]))
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


def _exact_score(s, case):
    parts = []
    for a in range(0, case["rows"], 256):
        x, token = s["logits"][a:a + 256].double(), s["token"][a:a + 256]
        order = torch.sort(x, dim=1, descending=True, stable=True).indices
        rank = (order == token[:, None]).int().argmax(1).int()
        best = order[:, :case["top"]]
        lp = torch.log_softmax(x * case["scale"], 1)
        entropy = -(torch.exp(lp) * lp.clamp(min=-1e300)).sum(1)
        parts.append((lp.gather(1, token[:, None]).squeeze(1), entropy, rank, lp.gather(1, best), best.int()))
    names = ("logprob", "entropy", "rank", "top_logprob", "top_index")
    return {name: torch.cat([p[i] for p in parts]) for i, name in enumerate(names)}
