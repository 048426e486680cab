"""Positions with several axes: ``append`` against its definition in 64 bits, and its refusals."""

import math
import os
import subprocess

import pytest
import torch

import kv_plain as P
from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import svfsim as S
from test_kvcache import BF, HF, batch_of, make
from test_kvcache_refusals import A, append, batch, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def axes(**kw):
    f = dict(kept=0, token=3, axis=1, axes=3, of_pair=bytes(128))
    f.update(kw)
    return C._AXES.pack(*f.values())


# -- on the CPU ------------------------------------------------------------------

@pytest.mark.parametrize("kw,args,text", [
    (dict(axes=0), {}, "axes"), (dict(axes=5), {}, "axes"), (dict(axes=2, of_pair=bytes([0, 1, 2])), {}, "of_pair"),
    (dict(of_pair=bytes(63) + b"\3"), {}, "of_pair"), (dict(token=-1), {}, "strides"), (dict(axis=1 << 41), {}, "strides"),
    ({}, dict(rot=7), "rot"), ({}, dict(rot=130), "rot"), ({}, dict(rope=0), "table"), ({}, dict(positions=0), "NULL"),
    ({}, dict(ot=2048), "in place"), ({}, dict(heads=7), "multiple of kv_heads"), ({}, dict(layout=2), "layout"),
])
def test_append_with_axes_refuses(kw, args, text):
    assert S.load().svf_kv_append_axes(cache(), batch(), append(**args), axes(**kw), None) == -1
    assert text in C.last_error()


def test_append_with_axes_needs_them_and_looks_at_the_pairs_that_there_are():
    lib = S.load()
    assert lib.svf_kv_append_axes(cache(), batch(), append(), None, None) == -1 and "axes" in C.last_error()
    # a pair behind the rotated part may say anything
    assert lib.svf_kv_append_axes(cache(), batch(num_tokens=0), append(rot=126), axes(of_pair=bytes(63) + b"\3"), None) == 0
    assert lib.svf_kv_append_axes(cache(num_pages=0), batch(num_tokens=1 << 26, num_seqs=1), append(heads=2), axes(), None) == -1


def test_struct_of_axes_has_the_headers_layout(tmp_path):
    src = tmp_path / "layout.c"
    src.write_text("""#include <stdio.h>
#include <stddef.h>
#include "svfkv.h"
int main(void) {
    printf("%zu %zu %zu %d\\n", sizeof(svf_kv_axes), offsetof(svf_kv_axes, axes), offsetof(svf_kv_axes, of_pair), SVF_KV_MOST_AXES);
    return 0;
}
""")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = list(map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()))
    assert got == [C._AXES.size, 24, 28, C.MOST_AXES]


def test_pair_axes():
    assert C.pair_axes((1, 3, 2)) == bytes([0, 1, 1, 1, 2, 2])
    assert C.pair_axes((1, 3, 2), "turns") == bytes([0, 1, 2, 1, 2, 1])
    assert C.pair_axes((4,)) == bytes(4) and C.pair_axes((0, 2)) == bytes([1, 1])
    for bad in ((), (1, 1, 1, 1, 1), (-1, 2), (100, 29)):
        with pytest.raises(S.SvfError):
            C.pair_axes(bad)
    with pytest.raises(S.SvfError):
        C.pair_axes((1, 2), "twice")


def test_rope_table_with_a_range_of_frequencies_for_each_axis():
    ax = C.pair_axes((8, 4, 4), "turns")
    t = C.rope_table(50, 32, base=100.0, device="cpu", axes=ax)
    for a, n in ((0, 8), (1, 4), (2, 4)):
        alone = C.rope_table(50, 2 * n, base=100.0, device="cpu")
        at = [i for i, x in enumerate(ax) if x == a]
        assert torch.equal(t[:, at], alone[:, :n]) and torch.equal(t[:, [i + 16 for i in at]], alone[:, n:])
    with pytest.raises(S.SvfError):
        C.rope_table(50, 30, device="cpu", axes=ax)


# -- on the GPU ------------------------------------------------------------------

def check(lens, new, pairs, order, layout, heads, kv_heads, dim, page, dtype, shift=0, n_axes=3, keep=True, seed=3, odd=True):
    """Runs append with axes and compares everything that it writes; returns the cache, queries and arguments."""
    s = make(20, lens, new, heads, kv_heads, dim, page, dtype, garbage=7.0, stats=True)
    g = torch.Generator().manual_seed(seed)
    T, n = sum(new), heads + 2 * kv_heads
    wide = torch.randn((T, n * dim + 8), generator=g).to(dtype)
    cut = lambda w: w[:, shift:shift + n * dim].view(T, n, dim)  # noqa: E731
    qkv = cut(wide)
    q, k, v = qkv.split((heads, kv_heads, kv_heads), 1)
    ax = C.pair_axes(pairs, order)
    half = len(ax)
    rot = 2 * half
    pos = torch.randint(0, 500, (T, n_axes), generator=g).int()
    kept = torch.randint(0, 9999, (T,), generator=g).int()
    if odd:
        pos[3, 0], pos[T - 1, n_axes - 1] = 500, -1                 # outside the table
    rope = C.rope_table(500, rot, device="cpu")
    cos, sin = torch.empty((T, half), dtype=torch.float64), torch.empty((T, half), dtype=torch.float64)
    for i, a in enumerate(ax):
        known = (pos[:, a] >= 0) & (pos[:, a] < 500)
        at = pos[:, a].clamp(0, 499).long()
        cos[:, i] = torch.where(known, rope[at, i].double(), math.nan)
        sin[:, i] = torch.where(known, rope[at, half + i].double(), math.nan)
    want_q, want_k = (P.rotate(x.double(), cos, sin, layout) for x in (q, k))
    kp, vp, wp, pp = s["k"].double(), s["v"].clone(), s["weight"].clone(), s["position"].clone()
    written = torch.zeros(kp.shape[:3], dtype=torch.bool)
    at = 0
    for i, m in enumerate(new):
        pg, row = P.slots_of(s["table"], i, lens[i], page, kp.shape[0])
        for t in range(m):
            j = lens[i] - m + t
            if j >= 0:
                kp[pg[j], :, row[j]], vp[pg[j], :, row[j]] = want_k[at + t], v[at + t]
                wp[pg[j], :, row[j]], pp[pg[j], :, row[j]] = 0.0, kept[at + t] if keep else pos[at + t, 0]
                written[pg[j], :, row[j]] = True
        at += m
    dev = wide.cuda()
    dq, dk, dv = cut(dev).split((heads, kv_heads, kv_heads), 1)
    c = C.Cache(s["k"].cuda(), s["v"].cuda(), s["weight"].cuda(), s["position"].cuda())
    more = dict(layout=layout, axes=ax, kept=kept.cuda() if keep else None)
    got = C.append(dq, dk, dv, pos.cuda(), rope.cuda(), batch_of(s), c, **more)
    u = P.UNIT[dtype]

    def near(x, y, size):       # two products and a sum in 32 bits, then one rounding to the type
        x = x.cpu().double()
        nan = y.isnan()
        assert torch.equal(x.isnan(), nan)
        assert ((x - y).abs() <= u * y.abs() * 1.01 + 2.0 ** -22 * size + 2.0 ** -25)[~nan].all()

    size = q.double().abs().max()
    near(got, want_q, size)
    near(c.k, kp, size)
    assert torch.equal(got[..., rot:].cpu(), q[..., rot:])
    assert torch.equal(c.k.cpu()[~written], s["k"][~written])
    assert torch.equal(c.v.cpu(), vp) and torch.equal(c.weight.cpu(), wp) and torch.equal(c.position.cpu(), pp)
    # in place of q, without weights and positions, and positions as rows of axes
    c2 = C.Cache(s["k"].cuda(), s["v"].cuda())
    rows = pos.t().contiguous().cuda()
    q2 = C.append(dq, dk, dv, rows.t(), rope.cuda(), batch_of(s), c2, q_out=dq, **more)
    assert q2.data_ptr() == dev.data_ptr() + shift * dev.element_size()
    assert torch.equal(torch.nan_to_num(q2, 9.0), torch.nan_to_num(got, 9.0))
    assert torch.equal(torch.nan_to_num(c2.k, 9.0), torch.nan_to_num(c.k, 9.0)) and torch.equal(c2.v, c.v)
    return s, c, got


PAIRS = [(64, (16, 8, 8)), (64, (3, 3, 3)), (64, (1, 1, 1)), (64, (5, 0, 27)), (128, (16, 24, 24)), (128, (24, 20, 20)),
         (128, (17, 5, 3)), (128, (1, 1, 2)), (128, (21, 21, 21)), (256, (32, 48, 48)), (256, (40, 41, 41)), (256, (9, 9, 9))]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,pairs", PAIRS)
@pytest.mark.parametrize("order", ["blocks", "turns"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("heads,kv_heads,shift", [(8, 2, 0), (5, 5, 0), (3, 1, 1)])
def test_append_with_axes(dtype, dim, pairs, order, layout, heads, kv_heads, shift):
    # two sequences have more tokens than slots
    check([5, 40, 1, 0, 17, 3], [5, 19, 1, 2, 0, 6], pairs, order, layout, heads, kv_heads, dim, 16, dtype, shift)


@pytest.mark.gpu
@pytest.mark.parametrize("n_axes,pairs", [(1, (64,)), (2, (32, 32)), (4, (16, 16, 16, 16)), (4, (7, 8, 9, 40))])
@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("page", [1, 64])
def test_append_with_one_to_four_axes(n_axes, pairs, keep, page):
    check([9, 130, 2], [4, 60, 1], pairs, "turns", "half", 4, 2, 128, page, BF, n_axes=n_axes, keep=keep)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [1, 2, 63, 64, 65, 1000, 5000])
def test_append_with_axes_of_few_and_many_tokens(tokens):
    check([tokens, tokens + 7], [tokens, 4], (16, 24, 24), "blocks", "half", 4, 1, 128, 16, BF, odd=tokens > 3)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (64, 40)])
def test_equal_positions_turn_as_one_axis_does(layout, dim, rot):
    """A text's tokens have the same position on every axis."""
    s = make(5, [30, 400], [30, 7], 8, 2, dim, 16, BF, stats=True)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((37, h, dim), generator=g).to(BF).cuda() for h in (8, 2, 2))
    pos = torch.randint(0, 900, (37,), generator=g).int().cuda()
    rope = C.rope_table(900, rot)
    one, three = ([C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position")))] for _ in range(2))
    a = C.append(q, k, v, pos, rope, batch_of(s), one[0], layout)
    third = rot // 6
    b = C.append(q, k, v, pos[:, None].expand(-1, 3), rope, batch_of(s), three[0], layout,
                 axes=C.pair_axes((rot // 2 - 2 * third, third, third)))
    near = lambda x, y: (x.double() - y.double()).nan_to_num(0.0).abs().max() <= 2.0 ** -7 * 5  # noqa: E731
    assert near(a, b) and near(one[0].k, three[0].k)
    assert torch.equal(one[0].position, three[0].position) and torch.equal(one[0].weight, three[0].weight)


@pytest.mark.gpu
def test_missing_pages_and_pages_outside_the_pool():
    s = make(6, [33, 40], [33, 8], 4, 2, 64, 16, BF, garbage=3.0, stats=True)
    s["table"][0, 1], s["table"][1, 2] = -1, s["k"].shape[0]
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((41, h, 64), generator=g).to(BF).cuda() for h in (4, 2, 2))
    pos = torch.zeros((41, 2), dtype=torch.int32, device="cuda")
    c = C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position")))
    before = c.v.clone()
    got = C.append(q, k, v, pos, C.rope_table(4, 32), batch_of(s), c, axes=C.pair_axes((8, 8)))
    assert torch.equal(got, q)                      # position 0 turns nothing
    table = s["table"]
    written = torch.zeros(before.shape[0], dtype=torch.bool)
    for p in (0, 2):
        written[table[0, p]] = True
    assert torch.equal(c.v[~written.cuda()], before[~written.cuda()])
    for j in list(range(16)) + [32]:
        assert torch.equal(c.v[table[0, j // 16], :, j % 16], v[j]) and torch.equal(c.k[table[0, j // 16], :, j % 16], k[j])


@pytest.mark.gpu
def test_append_with_axes_refuses_what_does_not_fit():
    s = make(7, [4], [4], 4, 2, 64, 16, BF, stats=True)
    q, k, v = (torch.zeros((4, h, 64), dtype=BF, device="cuda") for h in (4, 2, 2))
    c = C.Cache(s["k"].cuda(), s["v"].cuda())
    rope, ax = C.rope_table(8, 64), C.pair_axes((10, 11, 11))
    pos = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    kept = torch.zeros(4, dtype=torch.int32, device="cuda")
    for args, more, text in (((pos[:, 0], rope), dict(axes=ax), "tokens, axes"), ((pos.long(), rope), dict(axes=ax), "int32"),
                             ((pos, rope), dict(axes=ax[:-1]), "one for each pair"), ((pos, rope), dict(axes=list(ax)), "bytes"),
                             ((pos[:, :2], rope), dict(axes=ax), "of_pair"), ((pos, None), dict(axes=ax), "one for each pair"),
                             ((pos, rope), dict(axes=ax, kept=kept[:2]), "kept"), ((pos[:, 0].contiguous(), rope), dict(kept=kept), "kept"),
                             ((pos.expand(4, 3)[:3], rope), dict(axes=ax), "positions")):
        with pytest.raises(S.SvfError, match=text):
            C.append(q, k, v, *args, batch_of(s), c, **more)
