"""Scores of answers (``include/svflogprob.h``) on the GPU against their definition in 64 bits."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
INF, NAN = float("inf"), float("nan")


def plain(x, token, top, scale):
    """Row by row in 64 bits: (logprob, entropy, rank, top_logprob, top_index, tolerance of logprobs, of the
    entropy).  What is rounded: a logit's distance d from a reference, at most 6 from the largest, as a power of
    two (three roundings, 2^-24 each, of d), the exponential (2^-23), the sums (vocab / 256 + 64 additions one after
    another at most), logarithm and the last operations (2^-22)."""
    x = x.double()
    V = x.shape[1]
    y = torch.where(x.isnan(), -INF, x)
    order = torch.sort(y, dim=1, descending=True, stable=True).indices
    # NaN behind -inf: of those two alone the sort has mixed the order
    nan = x.isnan().gather(1, order)
    order = order.gather(1, torch.sort(nan.int(), dim=1, stable=True).indices)
    index = order[:, :top]
    known = (token >= 0) & (token < V)
    at = token.clamp(0, V - 1)[:, None]
    rank = torch.where(known, (order == at).int().argmax(1), -1)
    bad = (x.isnan() | (x == INF)).any(1)
    m = y.amax(1, keepdim=True)
    none = (m == -INF).squeeze(1) & ~bad
    d = torch.where(none[:, None] | bad[:, None], 0.0, (x - m) * scale)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    lp = torch.where(none[:, None], -INF, d - s.log())
    lp[bad] = NAN
    p = e / s
    dist = torch.where(p > 0, d.abs(), 0.0) + 6
    entropy = s.log().squeeze(1) - torch.where(p > 0, p * d, 0.0).sum(1)
    entropy = torch.where(none, 0.0, entropy)
    entropy[bad] = NAN
    steps = V / 256 + 64
    a, b = (p * dist).sum(1), (p * dist * dist).sum(1)
    lse = 2.0 ** -24 * (3 * a + steps) + 2.0 ** -22
    far = lp.abs().clamp(max=1e30)
    tol = lse[:, None] + 2.0 ** -24 * 4 * (torch.where(d.isfinite(), d.abs(), 0.0) + 6) + 2.0 ** -22 * far
    tol_entropy = lse + 2.0 ** -24 * (3 * b + (steps + 8) * a) + 2.0 ** -22 * entropy.abs()
    logprob = torch.where(known, lp.gather(1, at).squeeze(1), NAN)
    return logprob, entropy, rank, lp.gather(1, index), index, tol.gather(1, at).squeeze(1), tol.gather(1, index), tol_entropy


def near(got, want, tol):
    got = got.cpu().double()
    want = want.float().double()        # below -3.4e38 there is only -inf in 32 bits
    same = (got == want) | (got.isnan() & want.isnan())
    ok = same | ((got - want).abs() <= tol)
    assert ok.all(), (got[~ok][0], want[~ok][0], ok.logical_not().nonzero()[0].tolist())


def check(x, token, top=0, scale=1.0, dev=None):
    from paper_2606_22327_amd import logprobs as L
    r = L.score(x.cuda() if dev is None else dev, token.cuda(), top=top, scale=scale)
    lp, entropy, rank, top_lp, index, t0, t1, t2 = plain(x, token.long(), top, scale)
    assert r.rank.dtype == torch.int32 and r.top_index.dtype == torch.int32 and r.top_index.shape == (x.shape[0], top)
    assert r.logprob.dtype == r.entropy.dtype == r.top_logprob.dtype == F32
    assert torch.equal(r.rank.cpu().long(), rank)
    assert torch.equal(r.top_index.cpu().long(), index)
    near(r.logprob, lp, t0)
    near(r.entropy, entropy, t2)
    near(r.top_logprob, top_lp, t1)
    return r


def logits(seed, rows, vocab, dtype, size=3.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, vocab), generator=g) * size).to(dtype), torch.randint(0, vocab, (rows,), generator=g), g


VOCABS = [1, 2, 7, 8, 9, 63, 64, 65, 255, 257, 511, 2047, 2049, 4096, 5001, 16385, 50001, 131072]


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies(dtype, vocab):
    x, token, _ = logits(vocab, 5, vocab, dtype)
    check(x, token, top=min(vocab, 5))
    check(x, token.int(), top=min(vocab, 64))


@pytest.mark.parametrize("rows", [1, 2, 3, 17, 64, 255, 256, 257, 600])
@pytest.mark.parametrize("vocab", [700, 9001, 40000])
def test_numbers_of_rows(rows, vocab):
    x, token, _ = logits(rows, rows, vocab, BF)
    check(x, token, top=3)


@pytest.mark.parametrize("top", [0, 1, 2, 3, 20, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("rows,vocab", [(1, 30000), (300, 3001), (2, 150000)])
def test_numbers_of_alternatives(top, rows, vocab):
    x, token, _ = logits(top, rows, vocab, BF)
    check(x, token, top=top)
    check(x.float(), token, top=top)


@pytest.mark.parametrize("scale", [1 / 0.7, 0.25, 3.0, 1e-6, 50.0])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_temperatures(scale, dtype):
    x, token, _ = logits(1, 6, 20000, dtype)
    check(x, token, top=8, scale=scale)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("shift", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("pad", [0, 1, 6])
def test_rows_at_any_address(dtype, shift, pad):
    x, token, g = logits(2, 9, 5003, dtype)
    wide = torch.full((9 * (5003 + pad) + 8,), INF, dtype=dtype)       # between the rows: never read
    view = wide[shift:shift + 9 * (5003 + pad)].view(9, 5003 + pad)[:, :5003]
    view.copy_(x)
    dev = wide.cuda()[shift:shift + 9 * (5003 + pad)].view(9, 5003 + pad)[:, :5003]
    check(x, token, top=10, dev=dev)


def test_one_row_for_all():
    x, _, _ = logits(3, 1, 3000, BF)
    token = torch.arange(0, 3000, 100)
    check(x.expand(30, 3000), token, top=2, dev=x.cuda().expand(30, 3000))


def test_columns_apart_are_refused():
    from paper_2606_22327_amd import logprobs as L
    from paper_2606_22327_amd import svfsim as S
    x, token, _ = logits(3, 8, 8, BF)
    with pytest.raises(S.SvfError, match="contiguous in vocab"):
        L.score(x.cuda().t(), token.cuda())


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab,rows", [(3, 40), (5000, 11), (100001, 4), (100001, 1)])
def test_equal_logits_go_to_the_lowest_index(dtype, vocab, rows):
    g = torch.Generator().manual_seed(7)
    token = torch.randint(0, vocab, (rows,), generator=g)
    top = min(64, vocab)
    check(torch.zeros((rows, vocab), dtype=dtype), token, top=top)
    few = torch.randint(-1, 2, (rows, vocab), generator=g).to(dtype)
    check(few * 0.5, token, top=top)
    check(torch.where(few == 0, torch.tensor(-0.0, dtype=dtype), few * 0), token, top=top)     # -0 equals 0


@pytest.mark.parametrize("vocab", [4096, 70001])
@pytest.mark.parametrize("rows", [1, 40])
def test_rising_and_falling_rows_and_large_ones_at_every_distance(vocab, rows):
    i = torch.arange(vocab).float()
    token = torch.arange(rows) * 97 % vocab
    for x in (i / vocab, -i / vocab, torch.where(i % 8 == 3, 10.0 - i / vocab, i / vocab),
              torch.where(i % 2048 < 8, 5.0 + i / vocab, 0.0), torch.where(i % 256 == 0, 1.0, 0.0),
              torch.where(i % 1024 < 64, 20.0 + i % 7, 0.0)):
        check(x.expand(rows, vocab).contiguous(), token, top=64)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows", [1, 37])
def test_masked_rows(dtype, rows):
    x, token, g = logits(4, rows, 30011, dtype)
    lowest = torch.finfo(dtype).min
    hidden = torch.rand((rows, 30011), generator=g) < 0.9
    check(x.masked_fill(hidden, -INF), token, top=64)
    check(x.masked_fill(hidden, lowest), token, top=64)
    one = torch.full_like(x, -INF)
    one[torch.arange(rows), token] = 1.5                               # nothing but the token is allowed
    check(one, token, top=5)
    check(one, (token + 1) % 30011, top=5)
    r = check(torch.full_like(x, -INF), token, top=5)                  # nothing is
    assert (r.logprob == -INF).all() and (r.entropy == 0).all()
    check(torch.full_like(x, lowest), token, top=5)                    # all are equally unlikely
    check(torch.full_like(x, -lowest), token, top=5)
    x[:, 20000:] = -INF
    check(x, token, top=30)


@pytest.mark.parametrize("what", [NAN, -NAN, INF])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 21])
def test_rows_without_a_distribution(what, dtype, rows):
    x, token, g = logits(5, rows, 20003, dtype)
    x[::2, 11] = what
    x[::3, 20002] = what
    token[0] = 11
    r = check(x, token, top=9)
    assert r.logprob[0].isnan() and r.entropy[0].isnan()
    check(torch.full_like(x, NAN), token, top=9)
    y = torch.full_like(x, NAN)
    y[:, 100::200] = -INF                                              # NaN comes after -inf
    y[:, 777] = 3.0
    check(y, token, top=64)
    check(torch.full_like(x, INF), token, top=9)


def test_extreme_scales_of_logits():
    x, token, _ = logits(6, 5, 8000, F32)
    check(x * 1e30, token, top=7)
    check(x * 1e-30, token, top=7)
    check(x + 3e4, token, top=7)
    check(x - 3e4, token, top=7)
    check(x * 1e38, token, top=7)
    big = torch.zeros((2, 8000))
    big[:, 5000], big[:, 6000] = 3.4e38, -3.4e38
    check(big, torch.tensor([5000, 6000]), top=3, scale=2.0)
    check(big, torch.tensor([5000, 6000]), top=3, scale=1e-38)
    check(big, torch.tensor([6000, 1]), top=3, scale=0.3)
    low = torch.full((2, 8000), -3.4e38)
    low[:, 7000] = -3.3e38
    check(low, torch.tensor([7000, 1]), top=3)
    check(low, torch.tensor([7000, 1]), top=3, scale=1e-37)


def test_tokens_outside_the_vocabulary():
    x, token, _ = logits(8, 6, 5000, BF)
    for t in (token.int(), token.long()):
        t[0], t[1], t[2] = -1, 5000, -100
        r = check(x, t, top=2)
        assert r.rank[:3].tolist() == [-1, -1, -1] and r.logprob[:3].isnan().all() and not r.entropy.isnan().any()
    check(x, torch.full((6,), 2 ** 40), top=2)


def test_a_peak_first_or_last():
    """The running maximum rises at the end of a row, or never."""
    for at in (0, 1, 4999, 49990, 50000):
        x, token, _ = logits(9, 3, 50001, BF, 1.0)
        x[:, at] = 60.0
        token[0] = at
        check(x, token, top=2)


def test_no_rows():
    from paper_2606_22327_amd import logprobs as L
    r = L.score(torch.zeros((0, 100), dtype=BF, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), top=3)
    assert [tuple(t.shape) for t in r] == [(0,), (0,), (0,), (0, 3), (0, 3)]


def test_past_32_bit_offsets():
    """Rows behind 2^31 bytes and 2^31 elements of a buffer."""
    from paper_2606_22327_amd import logprobs as L
    rows, vocab = 70000, 40000
    big = torch.zeros((rows, vocab), dtype=BF, device="cuda")
    x, token, _ = logits(10, 3, vocab, BF)
    where = [0, 60000, rows - 1]
    big[where] = x.cuda()
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    t[where] = token.cuda()
    r = L.score(big, t, top=4)
    lp, entropy, rank, top_lp, index, t0, t1, t2 = plain(x, token, 4, 1.0)
    near(r.logprob[where], lp, t0)
    near(r.entropy[where], entropy, t2)
    assert torch.equal(r.rank[where].cpu().long(), rank) and torch.equal(r.top_index[where].cpu().long(), index)
    assert r.rank[1] == 0 and r.top_index[30000].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("rows,vocab,top", [(1, 128000, 20), (40, 50001, 5), (300, 5000, 64)])
def test_the_same_every_time_on_another_stream_and_in_a_graph(rows, vocab, top):
    from paper_2606_22327_amd import logprobs as L
    x, token, _ = logits(11, rows, vocab, BF)
    x, token = x.cuda(), token.cuda()
    want = L.score(x, token, top=top)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = L.score(x, token, top=top)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    y, t = torch.zeros_like(x), torch.zeros_like(token)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = L.score(y, t, top=top)
    other, to, _ = logits(12, rows, vocab, BF)
    for a, b in ((x, token), (other.cuda(), to.cuda()), (x, token)):
        y.copy_(a)
        t.copy_(b)
        want = L.score(a, b, top=top)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_logits_that_require_a_gradient_are_refused():
    from paper_2606_22327_amd import logprobs as L
    from paper_2606_22327_amd import svfsim as S
    x = torch.zeros((2, 10), device="cuda", requires_grad=True)
    t = torch.zeros(2, dtype=torch.int64, device="cuda")
    with pytest.raises(S.SvfError, match="backward"):
        L.score(x, t)
    with torch.no_grad():
        assert L.score(x, t).rank.tolist() == [0, 0]


# Few rows of many logits are split over workgroups, each of which may have its own kind of logits.

@pytest.mark.parametrize("dtype,vocab", [(BF, 128000), (HF, 131071), (F32, 90001)])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_parts_of_a_row(dtype, vocab, rows):
    x, token, g = logits(13, rows, vocab, dtype)
    lowest = torch.finfo(dtype).min
    at = torch.arange(vocab)
    for hidden in (at < vocab // 2, at >= vocab // 2, (at > 1000) & (at < vocab - 1000), at != 77777, at > 10):
        check(x.masked_fill(hidden, -INF), token, top=20)
        check(x.masked_fill(hidden, lowest), token, top=20)
    for where in (0, 5000, vocab // 2, vocab - 1):
        token = torch.full((rows,), where)
        check(x, token, top=3)
        for what in (NAN, INF, -INF):
            y = x.clone()
            y[0, where] = what
            check(y, token, top=3)
            check(y, (token + 1) % vocab, top=64)
    check(torch.zeros_like(x), token, top=64)
    steps = (at // (vocab // 7)).to(dtype).expand(rows, vocab).contiguous()
    check(steps, token, top=64)
    check(-steps, token, top=64)


def test_the_widest_vocabulary():
    vocab = 1 << 21
    x, token, _ = logits(14, 2, vocab, BF)
    token[0] = vocab - 1
    check(x, token, top=64)
    check(x.float(), token, top=64)


# Many short rows have two waves each, a long row to a CU has sixteen.

def short(rows, vocab, dtype):
    """A kind of row after the other: (logits, tokens)."""
    x, token, g = logits(15, rows, vocab, dtype)
    lowest, at = torch.finfo(dtype).min, torch.arange(vocab)
    kinds = [lambda y: y, lambda y: y.masked_fill(torch.rand(y.shape, generator=g) < 0.9, -INF),
             lambda y: y.masked_fill(torch.rand(y.shape, generator=g) < 0.9, lowest), lambda y: torch.full_like(y, -INF),
             lambda y: torch.full_like(y, lowest), lambda y: y * 0, lambda y: y.masked_fill(at == 11, NAN),
             lambda y: y.masked_fill(at == vocab - 1, INF), lambda y: y.masked_fill(at == 0, 60.0),
             lambda y: (at // 70).to(dtype).expand(y.shape), lambda y: (-at // 70).to(dtype).expand(y.shape),
             lambda y: torch.where(at % 200 == 100, -INF, NAN).to(dtype).expand(y.shape),
             lambda y: y.masked_fill(at >= 65, -INF), lambda y: y.masked_fill(at < vocab - 3, -INF)]
    for k, kind in enumerate(kinds):
        x[k::len(kinds)] = kind(x[k::len(kinds)])
    token[::9] = 0
    token[1::9] = vocab - 1
    token[2::9] = -1
    return x, token


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab", [1, 8, 65, 71, 1025, 2644, 4091, 4092, 8183, 8184])
def test_many_short_rows(dtype, vocab):
    x, token = short(513, vocab, dtype)
    check(x, token, top=min(vocab, 64))
    check(x, token, top=min(vocab, 3), scale=0.7)
    check(x, token)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("shift", [1, 4, 7])
def test_many_short_rows_at_any_address(dtype, shift):
    rows, vocab, stride = 600, 1231, 1234
    x, token = short(rows, vocab, dtype)
    wide = torch.full((rows * stride + 8,), INF, dtype=dtype)          # between the rows: never read
    wide[shift:shift + rows * stride].view(rows, stride)[:, :vocab].copy_(x)
    check(x, token, top=33, dev=wide.cuda()[shift:shift + rows * stride].view(rows, stride)[:, :vocab])


def test_many_short_rows_of_huge_logits():
    x, token, _ = logits(16, 520, 900, F32)
    for y in (x * 1e30, x * 1e38, x + 3e7, x * 1e-30):
        check(y, token, top=7)


@pytest.mark.parametrize("dtype,vocab", [(BF, 98312), (HF, 131001), (F32, 50001)])
@pytest.mark.parametrize("rows", [129, 256])
def test_a_long_row_to_a_workgroup(dtype, vocab, rows):
    x, token = short(rows, vocab, dtype)
    check(x, token, top=64)
    check(x, token, top=3)
    check(x, token)


def test_long_rows_at_any_address():
    rows, vocab, stride, shift = 131, 99001, 99003, 3
    x, token = short(rows, vocab, BF)
    wide = torch.full((rows * stride + 8,), INF, dtype=BF)             # between the rows: never read
    wide[shift:shift + rows * stride].view(rows, stride)[:, :vocab].copy_(x)
    check(x, token, top=33, dev=wide.cuda()[shift:shift + rows * stride].view(rows, stride)[:, :vocab])
