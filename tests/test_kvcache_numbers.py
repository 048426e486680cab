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
