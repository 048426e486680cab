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
