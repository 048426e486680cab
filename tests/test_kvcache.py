"""The paged cache's operators on the GPU against their plain forms in 64 bits."""

import math

import pytest
import torch

import kv_plain as P

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16


def make(seed, lens, new, heads, kv_heads, dim, page, dtype, spare=3, garbage=float("nan"), stats=False):
    """A pool with every sequence's slots in shuffled pages; what no slot holds is ``garbage``."""
    g = torch.Generator().manual_seed(seed)
    width = max([-(-x // page) for x in lens] + [1])
    need = [-(-x // page) for x in lens]
    pool = sum(need) + spare
    perm = torch.randperm(pool, generator=g)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)   # entries behind the length are never read
    k = torch.full((pool, kv_heads, page, dim), garbage, dtype=dtype)
    v = k.clone()
    at = 0
    for i, n in enumerate(lens):
        table[i, :need[i]] = perm[at:at + need[i]].int()
        at += need[i]
        pg, row = P.slots_of(table, i, n, page, pool)
        k[pg, :, row] = torch.randn((n, kv_heads, dim), generator=g).to(dtype)
        v[pg, :, row] = torch.randn((n, kv_heads, dim), generator=g).to(dtype)
    T = sum(new)
    s = {"k": k, "v": v, "table": table, "kv_len": torch.tensor(lens, dtype=torch.int32),
         "offsets": torch.tensor([0] + new).cumsum(0).int(), "max_q": max(new + [0]),
         "q": (torch.randn((T, heads, dim), generator=g) * 1.5).to(dtype)}
    if stats:
        s["weight"] = torch.rand((pool, kv_heads, page), generator=g)
        s["position"] = torch.zeros((pool, kv_heads, page), dtype=torch.int32)
    return s


def batch_of(s):
    from paper_2606_22327_amd import kvcache as C
    return C.Batch(s["offsets"].cuda(), s["kv_len"].cuda(), s["table"].cuda(), s["max_q"])


def check_attend(s, causal=True, window=0, scale=None, add_weight=False, q=None, k=None, v=None, max_rows=None):
    """Runs attend and compares everything it returns; returns what it returned."""
    from paper_2606_22327_amd import kvcache as C
    T, H, D = s["q"].shape
    sc = 1 / math.sqrt(D) if scale is None else scale
    out, lse, weight, tol = P.attend(s["q"], s["k"], s["v"], s["offsets"], s["kv_len"], s["table"], causal, window, sc)
    w = s["weight"].cuda() if add_weight else None
    cache = C.Cache(s["k"].cuda() if k is None else k, s["v"].cuda() if v is None else v, w)
    got, got_lse = C.attend(s["q"].cuda() if q is None else q, batch_of(s), cache, causal=causal, window=window,
                            scale=scale, add_weight=add_weight)
    assert got.dtype == s["q"].dtype and got.shape == s["q"].shape
    slots = int(s["kv_len"].max()) if len(s["kv_len"]) else 0
    x, e = got.cpu().double(), P.out_tolerance(s["q"].dtype, D, out, tol, slots)
    fine = torch.isfinite(out)
    bad = ~torch.where(fine, (x - out).abs() <= e, (x == out) | (x.isnan() & out.isnan()))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist(), x[bad][0], out[bad][0], e[bad][0])
    y = got_lse.cpu().double()
    empty = lse == -math.inf
    assert torch.equal(y == -math.inf, empty)
    ok = empty | ((y - lse).abs() <= P.lse_tolerance(D, lse, tol)) | (y.isnan() & lse.isnan())
    assert ok.all()
    if add_weight:
        z = w.cpu().double() - s["weight"].double()
        rows = s["max_q"] * H // s["k"].shape[1]
        assert ((z - weight).abs() <= P.weight_tolerance(D, s["weight"].double(), weight, tol, rows)).all()
    return got, got_lse, w


HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (4, 2, 256), (16, 1, 64), (24, 1, 128), (40, 1, 64), (20, 2, 256)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("page", [1, 16, 256])
def test_attend_single_tokens(dtype, heads, kv_heads, dim, page):
    s = make(1, [1, 17, 0, 64, 65, 300, 2, 128], [1, 1, 1, 1, 1, 1, 0, 1], heads, kv_heads, dim, page, dtype, stats=True)
    check_attend(s)
    check_attend(s, add_weight=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 37), (False, 5)])
def test_attend_chunks(dtype, heads, kv_heads, dim, causal, window):
    s = make(2, [150, 3, 1, 77, 40, 0, 200], [100, 3, 1, 2, 33, 5, 0], heads, kv_heads, dim, 16, dtype, stats=True)
    check_attend(s, causal=causal, window=window)
    check_attend(s, causal=causal, window=window, add_weight=True)


@pytest.mark.parametrize("new", [1, 2, 3, 5, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 129])
@pytest.mark.parametrize("heads,kv_heads,dim,page", [(4, 1, 128, 16), (2, 2, 64, 32), (6, 2, 128, 1), (4, 2, 256, 64)])
def test_attend_every_number_of_new_tokens(new, heads, kv_heads, dim, page):
    s = make(new, [new, new + 1, new + 130, max(new - 1, 0)], [new] * 4, heads, kv_heads, dim, page, BF, stats=True)
    check_attend(s, add_weight=True)


@pytest.mark.parametrize("length", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513, 1025])
@pytest.mark.parametrize("window", [0, 1, 32, 100])
def test_attend_lengths_and_windows(length, window):
    s = make(length, [length] * 3, [1, 2, 40], 8, 2, 128, 16, BF, stats=True)
    check_attend(s, window=window, add_weight=True)


def test_attend_rows_without_a_slot():
    # more new tokens than slots: the first rows see nothing; sequences of no slot at all
    s = make(5, [3, 0, 1, 30], [10, 4, 2, 70], 8, 2, 128, 16, BF, stats=True)
    out, lse, _ = check_attend(s, add_weight=True)
    assert (out[:7] == 0).all() and (lse[:7] == -math.inf).all()
    check_attend(s, window=1, add_weight=True)
    check_attend(s, causal=False, add_weight=True)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 6, 64, 63])
def test_attend_widest_windows(window):
    # as wide as the numbers go, and as the table: with more new tokens than slots among them
    s = make(24, [3, 0, 60, 64], [10, 4, 2, 64], 8, 2, 128, 16, BF, stats=True)
    check_attend(s, window=window, add_weight=True)
    s = make(25, [3, 0, 60, 64], [10, 4, 2, 1], 4, 2, 128, 16, BF, stats=True)
    check_attend(s, window=window, add_weight=True)


@pytest.mark.parametrize("new", [1, 2, 24, 90])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_attend_missing_pages_and_garbage(new, what):
    # pages that are not there in the middle, at the front and at the end; garbage everywhere else
    s = make(6, [100, 130, 95], [new] * 3, 8, 2, 128, 16, BF, garbage=what, stats=True)
    s["table"][0, 2] = -1
    s["table"][1, 0] = 1 << 30
    s["table"][2, 5] = s["k"].shape[0]
    check_attend(s, add_weight=True)
    check_attend(s, window=20, causal=False, add_weight=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [2, 3, 1, 4], [40, 90, 1, 70]])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1500)])
def test_attend_weights_where_most_slots_have_no_page(dtype, new, causal, window):
    # a pool of far fewer slots than the sequences' lengths: the last sequences' slots count as the first's
    lens = [1000, 2100, 500, 1400]
    s = make(23, lens, new, 8, 2, 128, 16, dtype, stats=True)
    keep = []
    for i, n in enumerate(lens):
        pages = -(-n // 16)
        for x in range(pages):
            if x in (1, pages // 2, pages - 1):
                keep.append(int(s["table"][i, x]))
                s["table"][i, x] = len(keep) - 1
            else:
                s["table"][i, x] = -1
    for x in ("k", "v", "weight", "position"):
        s[x] = s[x][keep].contiguous()
    check_attend(s, causal=causal, window=window, add_weight=True)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new,heads", [(2, 4), (4, 8), (8, 2), (40, 4), (100, 8)])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_attend_values_that_are_not_numbers_behind_the_mask(dtype, new, heads, what):
    # the last new token's key and value are not numbers: the rows before it do not see them
    s = make(7, [new + 61, new], [new, new], heads, 2, 128, 16, dtype, stats=True)
    for i in range(2):
        pg, row = P.slots_of(s["table"], i, int(s["kv_len"][i]), 16, s["k"].shape[0])
        s["v"][pg[-1], :, row[-1], 5:70] = what
        s["k"][pg[-1], 1, row[-1], 3] = float("nan")
    out, _, _ = check_attend(s)
    assert torch.isfinite(out[:new - 1]).all() and torch.isfinite(out[new:2 * new - 1]).all()
    # and a window that has passed them
    s = make(8, [new + 61, new + 40], [new, new], heads, 2, 128, 16, dtype)
    for i in range(2):
        pg, row = P.slots_of(s["table"], i, int(s["kv_len"][i]), 16, s["k"].shape[0])
        at = int(s["kv_len"][i]) - new
        s["v"][pg[at], 1, row[at], 5:70] = what
        s["v"][pg[at - 1], 0, row[at - 1], 1] = -what
    check_attend(s, window=max(new // 2, 1))


@pytest.mark.parametrize("new", [1, 40])
def test_attend_infinite_values_that_are_seen(new):
    s = make(9, [90], [new], 4, 2, 128, 16, BF)
    pg, row = P.slots_of(s["table"], 0, 90, 16, s["k"].shape[0])
    s["v"][pg[3], 0, row[3], 7] = float("inf")
    s["v"][pg[4], 0, row[4], 8] = -float("inf")
    s["v"][pg[5], 1, row[5], 9] = float("nan")
    out, _, _ = check_attend(s)
    assert (out[:, 0, 7] == math.inf).all() and (out[:, 0, 8] == -math.inf).all() and out[:, 2, 9].isnan().all()


@pytest.mark.parametrize("new", [1, 3, 50])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_attend_peaked_and_flat_scores(new, dtype):
    s = make(10, [333, 64], [new, new], 8, 2, 128, 16, dtype, stats=True)
    check_attend(s, scale=3.0, add_weight=True)
    check_attend(s, scale=0.0, add_weight=True)
    check_attend(s, scale=-0.5, add_weight=True)


@pytest.mark.parametrize("new", [1, 4, 70])
def test_attend_strides(new):
    """A pool kept row by row with all heads, queries inside a wider projection, one element off 16 bytes."""
    from paper_2606_22327_amd import kvcache as C
    s = make(11, [100, 75], [new, new], 8, 2, 128, 16, BF)
    pool = torch.full((s["k"].shape[0], 16, 5, 128), float("nan"), dtype=BF, device="cuda")
    pool[:, :, 1:3] = s["k"].transpose(1, 2).cuda()
    vpool = pool.clone()
    vpool[:, :, 2:4] = s["v"].transpose(1, 2).cuda()
    wide = torch.zeros((2 * new, 8 * 128 + 129), dtype=BF, device="cuda")
    q = wide[:, 1:1 + 1024].view(2 * new, 8, 128)
    q.copy_(s["q"])
    check_attend(s, q=q, k=pool[:, :, 1:3].transpose(1, 2), v=vpool[:, :, 2:4].transpose(1, 2))
    # an output inside a wider buffer
    buf = torch.zeros((2 * new, 12, 128), dtype=BF, device="cuda")
    cache = C.Cache(s["k"].cuda(), s["v"].cuda())
    want, _ = C.attend(s["q"].cuda(), batch_of(s), cache)
    C.attend(s["q"].cuda(), batch_of(s), cache, out=buf[:, 2:10])
    assert torch.equal(buf[:, 2:10], want) and (buf[:, :2] == 0).all() and (buf[:, 10:] == 0).all()


def test_attend_too_many_new_tokens_is_nan():
    from paper_2606_22327_amd import kvcache as C
    s = make(12, [30, 40], [3, 2], 8, 2, 128, 16, BF)
    s["max_q"] = 2
    out, lse = C.attend(s["q"].cuda(), batch_of(s), C.Cache(s["k"].cuda(), s["v"].cuda()))
    assert out[:3].isnan().all() and lse[:3].isnan().all()
    assert torch.isfinite(out[3:]).all()


def test_attend_shared_pages():
    # two sequences that begin with the same pages
    s = make(13, [64, 80], [1, 20], 8, 2, 128, 16, BF)
    s["table"][1, :3] = s["table"][0, :3]
    check_attend(s)


def test_attend_long_rows_are_split():
    s = make(14, [5000, 9001, 100], [1, 2, 1], 4, 1, 128, 16, BF, stats=True)
    a = check_attend(s, add_weight=True)
    s["max_q"] = 500
    s2 = make(15, [2300], [60], 4, 1, 128, 16, BF, stats=True)
    check_attend(s2, add_weight=True)
    # the same again: nothing depends on the order in which parts arrive
    from paper_2606_22327_amd import kvcache as C
    s["max_q"] = 2
    for _ in range(3):
        w = s["weight"].cuda()
        out, lse = C.attend(s["q"].cuda(), batch_of(s), C.Cache(s["k"].cuda(), s["v"].cuda(), w), add_weight=True)
        assert torch.equal(out, a[0]) and torch.equal(lse, a[1]) and torch.equal(w, a[2])


@pytest.mark.parametrize("dtype,heads,kv_heads,dim", [(BF, 8, 1, 128), (HF, 4, 2, 64), (BF, 4, 1, 256)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 700)])
def test_attend_few_row_tiles_are_split(dtype, heads, kv_heads, dim, causal, window):
    from paper_2606_22327_amd import kvcache as C
    s = make(18, [3000, 30, 1029, 0, 300], [40, 1, 70, 0, 33], heads, kv_heads, dim, 16, dtype, stats=True)
    s["table"][0, 50:55] = -1
    a = check_attend(s, causal=causal, window=window, add_weight=True)
    w = s["weight"].cuda()
    out, lse = C.attend(s["q"].cuda(), batch_of(s), C.Cache(s["k"].cuda(), s["v"].cuda(), w), causal=causal, window=window,
                        add_weight=True)
    assert torch.equal(out, a[0]) and torch.equal(lse, a[1]) and torch.equal(w, a[2])


@pytest.mark.parametrize("new", [1, 60])
def test_attend_parts_of_scores_that_are_not_numbers(new):
    # every key of some units and tiles, so that a part of a split row has no other scores
    s = make(21, [3000], [new], 4, 1, 128, 16, BF)
    pg, row = P.slots_of(s["table"], 0, 3000, 16, s["k"].shape[0])
    s["k"][pg[1024:1536], 0, row[1024:1536]] = float("nan")
    out, lse, _ = check_attend(s)
    assert out.isnan().all() and lse.isnan().all()


def test_attend_split_tiles_and_values_that_are_not_numbers():
    s = make(19, [2000], [60], 4, 1, 128, 16, BF)
    pg, row = P.slots_of(s["table"], 0, 2000, 16, s["k"].shape[0])
    s["v"][pg[100], 0, row[100], 7] = float("inf")
    s["v"][pg[1990], 0, row[1990], 9] = float("nan")
    out, _, _ = check_attend(s)
    assert (out[:, 0, 7] == math.inf).all() and torch.isfinite(out[:49, 0, 9]).all() and out[50:, 0, 9].isnan().all()


@pytest.mark.parametrize("new", [1, 64])
def test_attend_past_32_bit_offsets(new):
    """Pages whose elements lie past 2^32 bytes and 2^31 elements."""
    from paper_2606_22327_amd import kvcache as C
    s = make(16, [200], [new], 16, 8, 128, 16, BF)
    pages = 150000       # 2.46e9 elements each
    k = torch.empty((pages, 8, 16, 128), dtype=BF, device="cuda")
    v = torch.empty_like(k)
    used = s["table"][0].long()
    far = torch.tensor([pages - 1 - 7 * i for i in range(len(used))])
    k[far.cuda()], v[far.cuda()] = s["k"][used].cuda(), s["v"][used].cuda()
    want = C.attend(s["q"].cuda(), batch_of(s), C.Cache(s["k"].cuda(), s["v"].cuda()))
    s["table"][0] = far.int()
    got = C.attend(s["q"].cuda(), batch_of(s), C.Cache(k, v))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_attend_no_tokens_and_no_sequences():
    from paper_2606_22327_amd import kvcache as C
    s = make(17, [30, 40], [0, 0], 8, 2, 128, 16, BF)
    out, lse = C.attend(s["q"].cuda(), batch_of(s), C.Cache(s["k"].cuda(), s["v"].cuda()))
    assert out.shape == (0, 8, 128) and lse.shape == (0, 8)
    b = C.Batch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                torch.zeros((0, 4), dtype=torch.int32, device="cuda"), 1)
    C.attend(s["q"].cuda(), b, C.Cache(s["k"].cuda(), s["v"].cuda()))


def test_no_sequences_and_tables_without_a_page():
    from paper_2606_22327_amd import kvcache as C
    s = make(22, [30], [3], 8, 2, 128, 16, BF, stats=True)
    ints = dict(dtype=torch.int32, device="cuda")
    cache = C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position")))
    none = C.Batch(None, torch.zeros(0, **ints), torch.zeros((0, 4), **ints), 0)
    assert C.evict(none, cache, 8, 0, torch.zeros(0, **ints)).shape == (0,)
    # lengths are cut to what the table has: nothing
    b = C.Batch(torch.tensor([0, 1, 3], **ints), torch.tensor([5, 9], **ints), torch.zeros((2, 0), **ints), 2)
    out, lse = C.attend(s["q"].cuda(), b, cache, add_weight=True)
    assert (out == 0).all() and (lse == -math.inf).all()
    assert C.evict(b, cache, 4, 0, torch.tensor([5, 9], **ints)).tolist() == [0, 0]
    C.append(s["q"].cuda(), s["q"].cuda()[:, :2], s["q"].cuda()[:, :2], torch.zeros(3, **ints), None, b, cache)
    for x, n in zip(cache, ("k", "v", "weight", "position")):
        assert torch.equal(torch.nan_to_num(x.cpu().float()), torch.nan_to_num(s[n].float()))


# -- append --------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,rot,layout", [(128, 128, "half"), (128, 128, "interleaved"), (128, 64, "half"),
                                            (128, 32, "interleaved"), (64, 64, "half"), (256, 96, "interleaved"),
                                            (64, 10, "half"), (64, 6, "interleaved"), (128, 0, "half"), (128, 16, "half")])
@pytest.mark.parametrize("heads,kv_heads,shift", [(8, 2, 0), (5, 5, 0), (3, 1, 1)])
def test_append(dtype, dim, rot, layout, heads, kv_heads, shift):
    from paper_2606_22327_amd import kvcache as C
    lens, new, page = [5, 40, 1, 0, 17, 3], [5, 19, 1, 2, 0, 6], 16   # two sequences with more tokens than slots
    s = make(20, lens, new, heads, kv_heads, dim, page, dtype, garbage=7.0, stats=True)
    g = torch.Generator().manual_seed(3)
    T = sum(new)
    wide = torch.randn((T, (heads + 2 * kv_heads) * dim + 8), generator=g).to(dtype)
    qkv = wide[:, shift:shift + (heads + 2 * kv_heads) * dim].view(T, heads + 2 * kv_heads, dim)
    q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
    pos = torch.randint(0, 500, (T,), generator=g).int()
    pos[3], pos[-1] = 500, -1                                       # outside the table
    rope = C.rope_table(500, rot, device="cpu") if rot else None
    cos, sin = (torch.full((T, rot // 2), math.nan, dtype=torch.float64) for _ in range(2))
    known = (pos >= 0) & (pos < 500)
    if rot:
        cos[known], sin[known] = (x.double() for x in rope[pos[known].long()].split(rot // 2, 1))
    want_q, want_k = (P.rotate(x.double(), cos, sin, layout) for x in (q, k))
    kp, vp, wp, pp = s["k"].double(), s["v"].clone(), s["weight"].clone(), s["position"].clone()
    written = torch.zeros(kp.shape[:3], dtype=torch.bool)
    at = 0
    for i, n in enumerate(new):
        pg, row = P.slots_of(s["table"], i, lens[i], page, kp.shape[0])
        for t in range(n):
            j = lens[i] - n + t
            if j >= 0:
                kp[pg[j], :, row[j]], vp[pg[j], :, row[j]] = want_k[at + t], v[at + t]
                wp[pg[j], :, row[j]], pp[pg[j], :, row[j]] = 0.0, pos[at + t]
                written[pg[j], :, row[j]] = True
        at += n
    dev = wide.cuda()
    dq = dev[:, shift:shift + (heads + 2 * kv_heads) * dim].view(T, heads + 2 * kv_heads, dim)
    cache = C.Cache(s["k"].cuda(), s["v"].cuda(), s["weight"].cuda(), s["position"].cuda())
    args = (dq[:, heads:heads + kv_heads], dq[:, heads + kv_heads:], pos.cuda(), None if rope is None else rope.cuda(),
            batch_of(s), cache, layout)
    got = C.append(dq[:, :heads], *args)
    # a rotated element: two products and a sum in 32 bits, then one rounding to the type
    u = P.UNIT[dtype]

    def near(x, y, size):
        x = x.cpu().double()
        nan = y.isnan()
        assert torch.equal(x.isnan(), nan)
        assert ((x - y).abs() <= u * y.abs() * 1.01 + 2.0 ** -22 * size + 2.0 ** -25)[~nan].all()

    size = q.double().abs().max()
    near(got, want_q, size)
    near(cache.k, kp, size)
    assert torch.equal(got[..., rot:].cpu(), q[..., rot:])
    assert torch.equal(cache.k.cpu()[~written], s["k"][~written])
    assert torch.equal(cache.v.cpu(), vp) and torch.equal(cache.weight.cpu(), wp) and torch.equal(cache.position.cpu(), pp)
    # in place of q, and without weights and positions
    c2 = C.Cache(s["k"].cuda(), s["v"].cuda())
    q2 = C.append(dq[:, :heads], *args[:-2], c2, layout, q_out=dq[:, :heads])
    assert q2.data_ptr() == dq.data_ptr()
    assert torch.equal(torch.nan_to_num(q2, 9.0), torch.nan_to_num(got, 9.0))
    assert torch.equal(torch.nan_to_num(c2.k, 9.0), torch.nan_to_num(cache.k, 9.0)) and torch.equal(c2.v, cache.v)


@pytest.mark.parametrize("seqs", [1, 63, 64, 65, 300, 4097])
def test_append_finds_each_tokens_sequence(seqs):
    from paper_2606_22327_amd import kvcache as C
    g = torch.Generator().manual_seed(seqs)
    new = torch.randint(0, 3, (seqs,), generator=g)
    new[0] = 2
    lens = (new + torch.randint(0, 3, (seqs,), generator=g)).int()
    table = torch.randperm(seqs + 5, generator=g)[:seqs, None].int()
    T = int(new.sum())
    k = torch.randn((T, 1, 64), generator=g).to(BF).cuda()
    cache = C.Cache(*(torch.zeros((seqs + 5, 1, 8, 64), dtype=BF, device="cuda") for _ in range(2)))
    b = C.Batch(torch.cat((torch.zeros(1), new.cumsum(0))).int().cuda(), lens.cuda(), table.cuda(), 2)
    C.append(k, k, k + 1, torch.zeros(T, dtype=torch.int32, device="cuda"), None, b, cache)
    want = torch.zeros((seqs + 5, 8, 64), dtype=BF)
    at = 0
    for i in range(seqs):
        for t in range(int(new[i])):
            want[table[i, 0], int(lens[i] - new[i]) + t] = k[at, 0].cpu()
            at += 1
    assert torch.equal(cache.k[:, 0].cpu(), want)


def test_rope_table_scalings():
    from paper_2606_22327_amd import kvcache as C
    plain = C.rope_table(64, 64, device="cpu").double()
    i = torch.arange(32, dtype=torch.float64)
    angle = torch.arange(64, dtype=torch.float64)[:, None] * 10000.0 ** (-i / 32)
    assert (plain[:, :32] - angle.cos()).abs().max() < 2.0 ** -24 and (plain[:, 32:] - angle.sin()).abs().max() < 2.0 ** -24
    linear = C.rope_table(64, 64, scaling="linear", factor=4.0, device="cpu").double()
    assert (linear[:, :32] - (angle / 4).cos()).abs().max() < 2.0 ** -24
    base = C.rope_table(2, 64, scaling="base", factor=4.0, device="cpu").double()
    got = torch.asin(base[1, 32:])
    assert torch.isclose(got[31], angle[1, 31] / 4, rtol=1e-4) and torch.isclose(base[1, 0], angle[1, 0].cos(), rtol=1e-6)
    parts = C.rope_table(2, 64, scaling="by-parts", factor=4.0, original=4096, device="cpu").double()
    size = 0.1 * math.log(4.0) + 1
    got = torch.atan2(parts[1, 32:], parts[1, :32])
    assert torch.allclose(torch.hypot(parts[1, :32], parts[1, 32:]), torch.full((32,), size, dtype=torch.float64), rtol=1e-6)
    assert torch.isclose(got[0], angle[1, 0], rtol=1e-5) and torch.isclose(got[31], angle[1, 31] / 4, rtol=1e-4)
    assert ((got <= angle[1] * (1 + 1e-5)) & (got >= angle[1] / 4 * (1 - 1e-4))).all()


# -- evict ---------------------------------------------------------------------

def check_evict(s, budget, recent, first, after, kv_len=None):
    from paper_2606_22327_amd import kvcache as C
    kv_len = s["kv_len"] if kv_len is None else kv_len
    want = P.evict(s["k"], s["v"], s["weight"], s["position"], kv_len, s["table"], budget, recent, first, after)
    cache = C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position")))
    got = C.evict(C.Batch(None, kv_len.cuda(), s["table"].cuda(), 0), cache, budget, recent, after.cuda(), first=first)
    assert torch.equal(got.cpu(), want[4])
    for x, y in zip(cache, want):
        x = x.cpu()
        if x.dtype != torch.int32:
            assert torch.equal(x.isnan(), y.isnan())
            x, y = torch.nan_to_num(x), torch.nan_to_num(y)
        assert torch.equal(x, y)
    return cache, got


def evict_state(seed, lens, kv_heads, dim, page, dtype=BF):
    s = make(seed, lens, [1] * len(lens), kv_heads, kv_heads, dim, page, dtype, garbage=0.5, stats=True)
    g = torch.Generator().manual_seed(seed + 1)
    for i, n in enumerate(lens):
        pg, row = P.slots_of(s["table"], i, n, page, s["k"].shape[0])
        s["weight"][pg, :, row] = torch.exp(2 * torch.randn((n, kv_heads), generator=g))
        for h in range(kv_heads):
            s["position"][pg, h, row] = torch.randperm(n, generator=g).int() if h % 2 else torch.arange(n).int()
    return s


@pytest.mark.parametrize("lens,budget", [([33, 32, 31, 0, 100, 1], 32), ([1000, 1500, 64], 64), ([2, 3, 1], 1),
                                         ([700, 1025], 600), ([300], 299)])
@pytest.mark.parametrize("kv_heads,dim,page", [(2, 64, 16), (3, 128, 1), (1, 256, 64)])
def test_evict(lens, budget, kv_heads, dim, page):
    s = evict_state(30, lens, kv_heads, dim, page)
    after = torch.tensor(lens, dtype=torch.int32)
    check_evict(s, budget, 0, 0, after)
    check_evict(s, budget, budget // 2, min(4, budget // 2), after)
    check_evict(s, budget, budget, 0, after)


def test_evict_ties_and_values_that_are_not_numbers():
    lens = [200, 300]
    s = evict_state(31, lens, 2, 64, 16)
    after = torch.tensor(lens, dtype=torch.int32)
    s["weight"] = torch.randint(0, 3, s["weight"].shape, generator=torch.Generator().manual_seed(1)).float()
    check_evict(s, 128, 10, 2, after)
    s["weight"].zero_()
    s["weight"].view(-1)[::3] = -0.0
    check_evict(s, 128, 10, 2, after)
    s["weight"] = torch.randn(s["weight"].shape, generator=torch.Generator().manual_seed(2))
    flat = s["weight"].view(-1)
    flat[::5], flat[1::7], flat[2::11], flat[3::13] = math.nan, math.inf, -math.inf, 1e-42
    check_evict(s, 128, 10, 2, after)
    s["weight"].fill_(math.nan)
    check_evict(s, 128, 0, 0, after)


def test_evict_missing_pages_and_repeated_positions():
    lens = [200, 300]
    s = evict_state(32, lens, 2, 64, 16)
    after = torch.tensor(lens, dtype=torch.int32)
    s["table"][0, 3], s["table"][1, 12], s["table"][1, 1] = -1, 1 << 20, -5
    check_evict(s, 128, 10, 2, after)
    s["position"].zero_()
    check_evict(s, 128, 10, 2, after)
    check_evict(s, 128, 10, 0, torch.tensor([5, -2 ** 31], dtype=torch.int32))


def test_evict_more_slots_than_are_held_in_lds():
    lens = [33000]
    s = evict_state(33, lens, 1, 64, 256)
    s["weight"][:] = (s["weight"] * 4).round()        # ties
    check_evict(s, 31000, 64, 4, torch.tensor(lens, dtype=torch.int32))
    check_evict(s, 500, 64, 4, torch.tensor(lens, dtype=torch.int32))


@pytest.mark.parametrize("lens,budget", [([5000, 4960, 4000], 4950), ([5000, 100], 2000), ([4096], 3000), ([4097], 4000)])
def test_evict_either_way_of_moving_and_of_holding_keys(lens, budget):
    s = evict_state(35, lens, 2, 64, 64)
    check_evict(s, budget, 32, 4, torch.tensor(lens, dtype=torch.int32))


def test_evict_again_and_again():
    """Lengths handed back, tokens appended in between by hand: what a program does over many steps."""
    lens = [90, 64]
    s = evict_state(34, [128, 128], 2, 64, 16)
    kv_len, after = torch.tensor(lens, dtype=torch.int32), torch.tensor(lens, dtype=torch.int32)
    for step in range(4):
        cache, new = check_evict(s, 64, 16, 4, after, kv_len)
        s["k"], s["v"], s["weight"], s["position"] = (x.cpu() for x in cache)
        grown = new.cpu() + 20
        for i in range(2):
            pg, row = P.slots_of(s["table"], i, int(grown[i]), 16, s["k"].shape[0])
            for t in range(20):
                j = int(new[i]) + t
                s["weight"][pg[j], :, row[j]] = 0.1 * t
                s["position"][pg[j], :, row[j]] = int(after[i]) + t
        kv_len, after = grown.int(), after + 20


# -- together ------------------------------------------------------------------

def test_on_another_stream_and_recorded_into_a_graph():
    from paper_2606_22327_amd import kvcache as C
    s = make(40, [100, 75, 600], [1, 9, 1], 8, 2, 128, 16, BF, garbage=0.0, stats=True)
    s["position"][:] = torch.arange(s["position"].numel()).view_as(s["position"]).int()
    b = batch_of(s)
    rope = C.rope_table(1024, 128)
    pos = torch.arange(11, dtype=torch.int32, device="cuda")
    kn = torch.randn((11, 2, 128), device="cuda").to(BF)
    after = torch.tensor([100, 75, 600], dtype=torch.int32, device="cuda")
    start = [s[n].cuda() for n in ("k", "v", "weight", "position")]
    q = s["q"].cuda()

    def step(cache):
        qr = C.append(q, kn, kn, pos, rope, b, cache)
        out, lse = C.attend(qr, b, cache, add_weight=True)
        return qr, out, lse, C.evict(b, cache, 64, 8, after, first=2)

    cache = C.Cache(*(x.clone() for x in start))
    want = step(cache)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    other = C.Cache(*(x.clone() for x in start))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(other)
    side.synchronize()
    for x, y in zip((*want, *cache), (*got, *other)):
        assert torch.equal(x, y)
    held = C.Cache(*(x.clone() for x in start))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for x, y in zip(held, start):
            x.copy_(y)
        got = step(held)
    for _ in range(3):
        for x in (*got, *held):
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*want, *cache), (*got, *held)):
            assert torch.equal(x, y)
