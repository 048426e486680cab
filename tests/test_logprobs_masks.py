"""Scores of rows ruled out by finite numbers of any size, at any temperature."""

import pytest
import torch

from test_logprobs import BF, F32, HF, check, logits
from test_logprobs_many_candidates import masked

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [1.0, 1 / 1.5, 0.5, 0.01, 1e-6, 3.0])
@pytest.mark.parametrize("rows,vocab", [(1, 70001), (5, 32000), (270, 9001), (600, 409)])
def test_lowest_numbers_at_every_temperature(dtype, scale, rows, vocab):
    """A thread that meets ruled-out tokens alone must not spoil the sum: they add nothing where their distance is large."""
    for low in (torch.finfo(dtype).min, -1e30, -1e10, -3e9, -1e6):
        for allowed in (1, 7):
            x, token = masked(rows, vocab, dtype, low, allowed)
            check(x, token, top=3, scale=scale)
            check(x, (token + 5) % vocab, top=0, scale=scale)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [1e3, 1e6, 1e9, 1e20, 1e37])
@pytest.mark.parametrize("scale", [1.0, 0.3, 1e-3])
def test_logits_of_every_size(dtype, size, scale):
    x, token, g = logits(5, 40, 9001, F32, 1.0)
    x = (x * size).to(dtype)
    x[::2] = -x[::2].abs()
    y = torch.where(torch.rand(x.shape, generator=g) < 0.999, x, torch.randn(x.shape, generator=g).to(dtype))
    check(x, token, top=5, scale=scale)
    check(y, token, top=5, scale=scale)


def test_half_precision_at_every_temperature():
    for scale in (1.0, 0.5, 0.01, 20.0, 1e30):
        x, token = masked(270, 9001, HF, torch.finfo(HF).min, 3)
        check(x, token, top=5, scale=scale)
