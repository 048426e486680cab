"""Weights with a window and first tokens: where slots have no page, and where tokens also see those behind them."""

import pytest
import torch

from test_kvcache import BF, HF, make
from test_kvcache_first import check

pytestmark = pytest.mark.gpu


def thinned(seed, lens, new, heads, kv_heads, dim, page, dtype, keep):
    """Sequences of ``lens`` slots of which only the pages ``keep`` (from the end where negative) are there."""
    held = [sorted({x % -(-n // page) for x in keep}) for n in lens]
    s = make(seed, [len(h) * page for h in held], new, heads, kv_heads, dim, page, dtype, garbage=0.0, stats=True)
    g = torch.Generator().manual_seed(seed)
    s["k"], s["v"] = (torch.randn(s[x].shape, generator=g).to(dtype) for x in ("k", "v"))
    table = torch.full((len(lens), max(-(-n // page) for n in lens)), -1, dtype=torch.int32)
    for i, h in enumerate(held):
        table[i, h] = s["table"][i, :len(h)]
    s["table"], s["kv_len"] = table, torch.tensor(lens, dtype=torch.int32)
    return s


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads,kv_heads,dim,new", [(8, 2, 128, 1), (8, 2, 128, 5), (4, 4, 64, 1), (8, 2, 256, 3)])
@pytest.mark.parametrize("page", [1, 16, 64])
def test_few_rows_of_sequences_with_more_slots_than_the_pool(dtype, heads, kv_heads, dim, new, page):
    """There is room for the scores of as many slots as the pool has: those of most units here are formed again."""
    s = thinned(1, [6000, 4100, 5000, 700], [new, 1, new, 1], heads, kv_heads, dim, page, dtype, (0, 1, 2, 33, 41, -20, -9, -2, -1))
    for window, first in ((4000, 100), (3000, 7), (6000, 40)):
        a = check(s, window, first, add_weight=True)
        b = check(s, window, first, add_weight=True)
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        check(s, window, first, causal=False, add_weight=True)


@pytest.mark.parametrize("heads,kv_heads,dim,lens,new,window,first", [
    (8, 2, 128, [2500], [2500], 100, 4), (4, 1, 64, [1900, 40, 1500], [1900, 1, 1200], 300, 70), (8, 1, 128, [1300], [1000], 64, 600),
    (2, 2, 256, [1500, 900], [1400, 900], 16, 1), (16, 2, 128, [3000, 2000], [700, 30], 50, 300)])
def test_prompts_whose_tokens_see_what_is_behind_them(heads, kv_heads, dim, lens, new, window, first):
    """Not causal: a slot tile of the window is met by every row before it too."""
    s = make(2, lens, new, heads, kv_heads, dim, 16, BF, stats=True)
    _, _, a = check(s, window, first, causal=False, add_weight=True)
    _, _, b = check(s, window, first, causal=False, add_weight=True)
    assert torch.equal(a, b)
