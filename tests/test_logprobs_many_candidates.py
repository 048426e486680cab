"""Scores of rows in which very many logits could be among the best: masked by a finite number, equal, in blocks."""

import pytest
import torch

from test_logprobs import BF, F32, HF, INF, check, logits

pytestmark = pytest.mark.gpu


def masked(rows, vocab, dtype, low, allowed, seed=1):
    g = torch.Generator().manual_seed(seed)
    x = torch.full((rows, vocab), low, dtype=dtype)
    at = torch.stack([torch.randperm(vocab, generator=g)[:allowed] for _ in range(rows)])
    return x.scatter_(1, at, torch.randn((rows, allowed), generator=g).to(dtype)), at[:, 0].clone()


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 128000), (3, 70001), (300, 20011), (600, 4001)])
@pytest.mark.parametrize("allowed", [1, 3, 40])
def test_masked_by_a_finite_number(dtype, rows, vocab, allowed):
    for low in (torch.finfo(dtype).min, -1e4):
        x, token = masked(rows, vocab, dtype, low, allowed)
        check(x, token, top=20)
        check(x, (token + 1) % vocab, top=64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 270])
@pytest.mark.parametrize("low", [-INF, -1e4])
def test_a_block_of_tokens_is_allowed(dtype, rows, low):
    """As many as some pieces of the row have, all others ruled out."""
    x, token, _ = logits(2, rows, 50001, dtype)
    for begin, end in ((10000, 18192), (0, 3001), (47000, 50001)):
        y = torch.full_like(x, low)
        y[:, begin:end] = x[:, begin:end]
        check(y, token, top=64)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 70001), (270, 30003), (600, 3001)])
def test_equal_rows_and_rows_without_a_distribution(dtype, rows, vocab):
    x, token, g = logits(3, rows, vocab, dtype)
    check(torch.zeros_like(x), token, top=64)
    y = x.clone()
    y[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] = float("nan")
    check(y, token, top=64)
    y[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] = INF
    check(y, token, top=64)
    check(torch.full_like(x, float("nan")), token, top=64)
    y = torch.full_like(x, float("nan"))
    y[:, ::3] = -INF
    y[:, 5] = 1.0
    check(y, token, top=64)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("threads", [128, 512, 1024])
def test_large_logits_that_one_thread_meets(dtype, threads):
    """In steps of what a workgroup of so many threads takes at a time: more of them than there is room for."""
    W = 4 if dtype == F32 else 8
    vocab = min(threads * W * (2300 // W), (1 << 20) + 77)
    x = torch.zeros((1, vocab), dtype=dtype)
    i = torch.arange(vocab)
    x[0, (i % (threads * W)) < W] = 5.0
    x[0, i[(i % (threads * W)) < W][100:]] = 6.0
    check(x, torch.tensor([vocab // 2]), top=64)
    rows = 257      # one part, and so in one workgroup
    r = check(x, torch.tensor([vocab // 2]), top=64)
    from paper_2606_22327_amd import logprobs as L
    many = L.score(x.cuda().expand(rows, vocab), torch.full((rows,), vocab // 2).cuda(), top=64)
    assert torch.equal(many.top_index, r.top_index.expand(rows, 64)) and torch.equal(many.rank, r.rank.expand(rows))


def test_a_finite_mask_costs_no_more_than_some_passes():
    """Constrained decoding: three allowed tokens of 128,000.  Ruled out by the type's lowest number, a call may take a few times what it
    takes where they are ruled out by -infinity (a pass for each alternative is 20 and 60 times)."""
    from paper_2606_22327_amd import logprobs as L
    low = torch.finfo(BF).min
    x, token = masked(203, 128000, BF, low, 3)
    x, token = x.cuda(), token.cuda()
    y = x.masked_fill(x == low, -INF)

    def least(x, top):
        times = []
        for _ in range(6):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(3):
                L.score(x, token, top=top)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    for top in (20, 64):
        assert least(x, top) < 5 * least(y, top), top
