"""Weights with a window and first tokens: where slots have no page, and where tokens also see those behind them."""

import pytest
import torch

from test_kvcache import BF, make
from test_kvcache_first import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,dim,lens,new,window,first", [
    (8, 2, 128, [2500], [2500], 100, 4), (4, 1, 64, [1900, 40, 1500], [1900, 1, 1200], 300, 70), (8, 1, 128, [1300], [1000], 64, 600),
    (2, 2, 256, [1500, 900], [1400, 900], 16, 1), (16, 2, 128, [3000, 2000], [700, 30], 50, 300)])
def test_prompts_whose_tokens_see_what_is_behind_them(heads, kv_heads, dim, lens, new, window, first):
    """Not causal: a slot tile of the window is met by every row before it too."""
    s = make(2, lens, new, heads, kv_heads, dim, 16, BF, stats=True)
    _, _, a = check(s, window, first, causal=False, add_weight=True)
    _, _, b = check(s, window, first, causal=False, add_weight=True)
    assert torch.equal(a, b)
