"""Numbers at their edges in the paged cache's operators: infinities, values that are no numbers, probabilities far
below a row's largest, and the bits that outputs keep."""

import math

import pytest
import torch

import kv_plain as P
from test_kvcache import check_attend, make

BF, HF = torch.bfloat16, torch.float16


def far_below(seed, length, new, dtype, slot, what):
    """Every row sees ``slot`` with a score 200 below the others', which is a probability of 1e-87, and one of its values is ``what``."""
    s = make(seed, [length], [new], 4, 1, 64, 16, dtype)
    pg, row = P.slots_of(s["table"], 0, length, 16, s["k"].shape[0])
    s["q"][..., 0] = 8
    s["k"][pg[slot], 0, row[slot], 0] = -200
    s["v"][pg[slot], 0, row[slot], 7] = what
    return s


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("length,new", [(100, 1), (300, 40), (300, 100)])
@pytest.mark.parametrize("what", [math.inf, -math.inf, math.nan])
def test_infinite_values_reach_every_row_that_sees_them(dtype, length, new, what):
    out, _, _ = check_attend(far_below(50, length, new, dtype, 5, what))
    assert out[..., 7].isnan().all() if math.isnan(what) else (out[..., 7] == what).all()
    assert torch.isfinite(out[..., :7]).all() and torch.isfinite(out[..., 8:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 64), (4, 1, 128), (4, 2, 256)])
@pytest.mark.parametrize("length,new", [(700, 1), (700, 8), (700, 100), (3000, 40)])
def test_outputs_keep_their_bits_whatever_the_number_of_rows(dtype, heads, kv_heads, dim, length, new):
    """The output is rounded to the type, the probabilities are not: as two numbers of the type they keep 2^-15 of themselves in
    bfloat16 (8 bits of what 8 bits leave) and 2^-21 in float16.  The rest as in ``out_tolerance``."""
    s = make(51, [length], [new], heads, kv_heads, dim, 16, dtype)
    out, _, _, tol = P.attend(s["q"], s["k"], s["v"], s["offsets"], s["kv_len"], s["table"], True, 0, dim ** -0.5)
    got, _, _ = check_attend(s)
    kept = P.out_tolerance(dtype, dim, out, tol, length) - 1.01 * P.UNIT[dtype] * tol["absv"]
    kept = kept + (2.0 ** -15 if dtype == BF else 2.0 ** -21) * tol["absv"]
    assert ((got.cpu().double() - out).abs() <= kept).all()


def added_weights(s, causal, window):
    """What attention adds to each slot's weight, in 64 bits: the softmax of every row over the slots that it sees, and of no others."""
    q, k, (T, H, D) = s["q"].double(), s["k"].double(), s["q"].shape
    pages, hk, page = k.shape[:3]
    weight = torch.zeros((pages, hk, page), dtype=torch.float64)
    for i in range(len(s["kv_len"])):
        a, b = int(s["offsets"][i]), int(s["offsets"][i + 1])
        pg, row = P.slots_of(s["table"], i, s["kv_len"][i], page, pages)
        j = torch.arange(len(pg))
        for t in range(a, b):
            own = len(pg) - (b - t)
            w = (pg >= 0) & (j <= own if causal else j >= 0) & (j > own - window if window else j >= 0)
            for h in range(H):
                g = h // (H // hk)
                x = D ** -0.5 * (k[pg[w], g, row[w]] @ q[t, h])
                e = torch.exp(x - x.max()) if len(x) else x
                weight[pg[w], g, row[w]] += e / e.sum()
    return weight


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [1, 4, 8, 40])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 30)])
@pytest.mark.parametrize("what", ["query", "key", "infinite key", "first slot's key"])
def test_weights_of_rows_that_are_not_numbers_stay_with_the_slots_they_see(dtype, new, causal, window, what):
    """A row whose statistic is no number, in a sequence whose table is filled up with another's pages: that one's weights, and those
    of slots which the row does not see, are what they are without it."""
    from paper_2606_22327_amd import kvcache as C
    s = make(52, [100, 75, 200, 40], [new] * 4, 8, 2, 64, 16, dtype, stats=True)
    tol = P.attend(s["q"], s["k"], s["v"], s["offsets"], s["kv_len"], s["table"], causal, window, 64 ** -0.5)[3]
    for i in (0, 1, 3):
        used = -(-int(s["kv_len"][i]) // 16)
        s["table"][i, used:] = s["table"][2, 3:3 + s["table"].shape[1] - used]
    pg, row = P.slots_of(s["table"], 1, 75, 16, s["k"].shape[0])
    if what == "query":
        s["q"][2 * new - 1, 5, 7] = math.nan
    else:
        at = {"key": 74, "infinite key": 73 if new > 1 else 74, "first slot's key": 75 - new}[what]
        s["k"][pg[at], 1, row[at], 3] = math.inf if what == "infinite key" else math.nan
    add = added_weights(s, causal, window)
    w = s["weight"].cuda()
    C.attend(s["q"].cuda(), C.Batch(s["offsets"].cuda(), s["kv_len"].cuda(), s["table"].cuda(), new),
             C.Cache(s["k"].cuda(), s["v"].cuda(), w), causal=causal, window=window, add_weight=True)
    z = w.cpu().double() - s["weight"].double()
    assert torch.equal(z.isnan(), add.isnan()) and add.isnan().any() and not add.isnan().all()
    ok = (z - add).abs() <= P.weight_tolerance(64, s["weight"].double(), add, tol, 4 * new)
    assert (ok | add.isnan()).all()


@pytest.mark.parametrize("rot,base,original", [(128, 10000.0, 4096), (128, 10000.0, 65536), (64, 500000.0, 8192), (128, 10000.0, 262144),
                                               (64, 10000.0, 100), (32, 10000.0, 5), (64, 10000.0, 3000000)])
def test_rope_by_parts_follows_its_turns_for_short_and_long_contexts(rot, base, original):
    """Pairs by their turns within the original context: more than ``fast`` stay, fewer than ``slow`` are divided by the factor, and between
    them there is one straight ramp, wherever it ends.  (Angles of position 1 from the table: 2^-24 of rounding.)"""
    from paper_2606_22327_amd import kvcache as C
    factor, fast, slow = 4.0, 32.0, 1.0
    t = C.rope_table(2, rot, base=base, scaling="by-parts", factor=factor, original=original, device="cpu").double()
    freq = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    part = (1 - torch.atan2(t[1, rot // 2:], t[1, :rot // 2]) / freq) / (1 - 1 / factor)      # 0: stays, 1: divided
    err = 2.0 ** -22 / freq
    turns = original * freq / (2 * math.pi)
    assert (part.abs() <= err)[turns >= fast].all() and ((part - 1).abs() <= err)[turns <= slow].all()
    step = 2 * math.log(base) / rot                     # in ln turns, from a pair to the next
    x = torch.log(turns) / step                         # falls by one a pair
    # the ramp begins at the last pair position that turns at least fast, and ends at the first that turns at most slow
    lo = math.floor(x[0].item() - math.log(fast) / step + 1e-9)
    hi = math.ceil(x[0].item() - math.log(slow) / step - 1e-9)
    want = ((torch.arange(rot // 2, dtype=torch.float64) - lo) / (hi - lo)).clamp(0, 1)
    assert ((part - want).abs() <= err).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("slot", [5, 1500, 2900])
@pytest.mark.parametrize("what", [math.inf, -math.inf])
def test_infinite_values_pass_the_join_of_split_rows(dtype, new, slot, what):
    """The part that has the value has scores far below the others', so that its factor becomes 0."""
    s = far_below(53, 3000, new, dtype, slot, what)
    pg, row = P.slots_of(s["table"], 0, 3000, 16, s["k"].shape[0])
    part = torch.arange(3000) // 500 == slot // 500
    s["k"][pg[part], 0, row[part], 0] = -200
    out, _, _ = check_attend(s)
    assert (out[..., 7] == what).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("length", [100, 3000])
@pytest.mark.parametrize("new", [1, 40])
def test_rows_of_infinitely_small_scores_are_zero_whatever_their_values(dtype, length, new):
    from paper_2606_22327_amd import kvcache as C
    s = far_below(54, length, new, dtype, 5, math.inf)
    s["k"][..., 0] = -math.inf
    out, lse = C.attend(s["q"].cuda(), C.Batch(s["offsets"].cuda(), s["kv_len"].cuda(), s["table"].cuda(), new),
                        C.Cache(s["k"].cuda(), s["v"].cuda()))
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("length,new", [(100, 1), (3000, 1), (300, 40), (3000, 40)])
def test_values_at_the_types_limit(dtype, length, new):
    """Means of the type's largest numbers are finite, sums before they are divided must be as well."""
    s = make(55, [length], [new], 4, 1, 64, 16, dtype)
    pg, row = P.slots_of(s["table"], 0, length, 16, s["k"].shape[0])
    s["v"][pg, 0, row, 7] = torch.finfo(dtype).max
    s["v"][pg, 0, row, 8] = torch.finfo(dtype).min
    out, _, _ = check_attend(s)
    assert (out[..., 7] == torch.finfo(dtype).max).all() and (out[..., 8] == torch.finfo(dtype).min).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("length,new,window", [(700, 1, 0), (700, 100, 0), (3000, 40, 0), (3000, 40, 900), (700, 100, 100)])
def test_values_that_are_no_numbers_all_over(dtype, length, new, window):
    """Whole dimensions of them, of one kind and of two, over tiles that all rows see and tiles that some do not."""
    s = make(56, [length], [new], 4, 1, 128, 16, dtype)
    pg, row = P.slots_of(s["table"], 0, length, 16, s["k"].shape[0])
    for d, what in ((3, math.nan), (4, math.inf), (77, -math.inf)):
        s["v"][pg, 0, row, d] = what
    s["v"][pg[::2], 0, row[::2], 126] = math.inf
    s["v"][pg[1::2], 0, row[1::2], 126] = -math.inf
    out, _, _ = check_attend(s, window=window)
    assert out[..., 3].isnan().all() and (out[..., 4] == math.inf).all() and (out[..., 77] == -math.inf).all() and out[..., 126].isnan().all()
    assert torch.isfinite(out[..., :3]).all() and torch.isfinite(out[..., 127]).all()
