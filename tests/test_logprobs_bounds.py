"""What no rounding may take from scores of answers: a probability is at most 1, an entropy at least 0."""

import math

import pytest
import torch

from test_logprobs import BF, F32, HF, INF, check, logits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("rows,vocab", [(400, 1000), (300, 32000), (2, 150000)])
@pytest.mark.parametrize("scale", [1.0, 1 / 0.7])
def test_one_allowed_token_is_certain(dtype, rows, vocab, scale):
    """All others at -infinity: ln 1 = 0, whatever the one logit is.  The sum is a power of two times its inverse, a step of
    2^-23 each and half a one for the product, and its logarithm has a step: below 2^-21."""
    from paper_2606_22327_amd import logprobs as L
    _, token, g = logits(rows, rows, vocab, F32)
    x = torch.full((rows, vocab), -INF, dtype=dtype)
    x[torch.arange(rows), token] = (10 * torch.randn(rows, generator=g)).to(dtype)
    r = L.score(x.cuda(), token.cuda(), top=2, scale=scale)
    for y in (r.logprob, -r.entropy, r.top_logprob[:, 0]):
        assert (y <= 0).all() and (y >= -2.0 ** -21).all(), (y.max(), y.min())
    assert (r.top_logprob[:, 1] == -INF).all() and torch.equal(r.top_index[:, 0].cpu().long(), token)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ahead", [8.0, 20.0, 40.0, 120.0])
@pytest.mark.parametrize("rows,vocab", [(300, 5001), (3, 150000)])
def test_near_certain_tokens(dtype, ahead, rows, vocab):
    x, token, _ = logits(int(ahead), rows, vocab, dtype, 1.0)
    x[torch.arange(rows), token] += ahead
    r = check(x, token, top=5)
    assert (r.logprob <= 0).all() and (r.top_logprob <= 0).all() and (r.entropy >= 0).all()


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("vocab", [131072, 1 << 20])
@pytest.mark.parametrize("at", [0, 5000, 77777])
def test_a_likely_token_does_not_swallow_the_others(dtype, vocab, at):
    """One token at 0 and all others at -25 powers of two: each of those is half a step of the sum that has the one, all of them
    together are 2^-8 or 2^-5 of it.  Of a logit's way into the sum: W - 1 additions in its 16 bytes, 4 of those, one for each time
    that a thread of 512 comes by with its 4, and 15 over the workgroup, 2^-24 each; exponentials, their distance and the logarithm less
    than 2^-21 together; in the entropy each of it twice, and distances of 25 rounded to 2^-20."""
    from paper_2606_22327_amd import logprobs as L
    x = torch.full((1, vocab), -25.0).to(dtype)
    x[0, at] = 0.0
    scale = torch.tensor(math.log(2.0)).item()          # in 32 bits
    r = L.score(x.cuda().expand(257, vocab), torch.full((257,), at).cuda(), scale=scale)
    W = 4 if dtype == F32 else 8
    tol = (W - 1 + 4 + vocab / (512 * 4 * W) + 15) * 2.0 ** -24 + 2.0 ** -21
    e = (vocab - 1) * math.exp(-25 * scale)
    want, entropy = -math.log1p(e), math.log1p(e) + 25 * scale * e / (1 + e)
    assert (r.logprob.double() - want).abs().max() <= tol, (r.logprob[0].item() - want, tol)
    assert (r.entropy.double() - entropy).abs().max() <= 2 * tol + 2.0 ** -20 * 25 * e
