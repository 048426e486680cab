"""Ends of ranges and equalities that are held exactly: the smallest scale, a workspace that there must be, equal positions."""

import math

import pytest
import torch

import kv_plain as P
from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import logprobs as L
from paper_2606_22327_amd import svfsim as S
from test_kvcache import BF, HF, batch_of, make
from test_logprobs_refusals import A, args

SMALLEST = 2.0 ** -149      # of what 32 bits hold above 0


def test_the_smallest_scale_is_one():
    lib = S.load()
    assert lib.svf_logprob(args(rows=0, scale=SMALLEST), None) == 0
    assert lib.svf_logprob(args(rows=0, scale=-SMALLEST), None) == -1 and "scale" in L.last_error()
    assert lib.svf_logprob(args(rows=0, scale=2.0 ** 126), None) == -1 and "scale" in L.last_error()


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_a_row_in_parts_needs_a_workspace(dtype):
    lib, kw = S.load(), dict(rows=1, vocab=150000, dtype=dtype)
    need = lib.svf_logprob_workspace(args(**kw))
    assert need > 0
    for more in (dict(workspace_bytes=need - 1), dict(workspace=A + 16), dict(workspace=0)):
        assert lib.svf_logprob(args(**kw, **more), None) == -1 and "workspace" in L.last_error()
    assert lib.svf_logprob_workspace(args(rows=4000, vocab=2000, dtype=dtype)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [3, 5001, 150000])
def test_at_the_smallest_scale_all_tokens_are_alike(vocab):
    """Logits up to 3e38 differ by less than 2^-20 once scaled: ln p is -ln vocab to that, a step of it and the sum's steps."""
    g = torch.Generator().manual_seed(1)
    x = (2 * torch.rand((2, vocab), generator=g) - 1) * 3e38
    r = L.score(x.cuda(), torch.tensor([0, vocab - 1]).cuda(), top=3, scale=SMALLEST)
    tol = 2.0 ** -20 + 2.0 ** -22 * math.log(vocab) + (vocab / 256 + 64) * 2.0 ** -24
    for y in (r.logprob, -r.entropy, r.top_logprob):
        assert (y.double() + math.log(vocab)).abs().max() <= tol
    assert torch.equal(r.top_index.cpu().long(), x.topk(3, 1).indices)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (64, 40)])
def test_a_texts_tokens_turn_as_with_one_axis(dtype, layout, dim, rot):
    """The same position on every axis: both ways are the same rotation but for one rounding each, and nothing is NaN but slots
    that nobody wrote."""
    s = make(5, [30, 400], [30, 7], 8, 2, dim, 16, dtype, stats=True)
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((37, h, dim), generator=g).to(dtype).cuda() for h in (8, 2, 2))
    pos = torch.randint(0, 900, (37,), generator=g).int().cuda()
    rope, third = C.rope_table(900, rot), rot // 6
    one, three = (C.Cache(*(s[n].cuda() for n in ("k", "v", "weight", "position"))) for _ in range(2))
    a = C.append(q, k, v, pos, rope, batch_of(s), one, layout)
    b = C.append(q, k, v, pos[:, None].expand(-1, 3), rope, batch_of(s), three, layout,
                 axes=C.pair_axes((rot // 2 - 2 * third, third, third)))
    assert not a.isnan().any() and not b.isnan().any()
    # a pair's length is at most 8; each side is rounded in 32 bits thrice and once to the type
    near = lambda x, y: ((x.double() - y.double()).abs() <= 2 * P.UNIT[dtype] * y.double().abs() + 2.0 ** -19).all()  # noqa: E731
    assert near(a, b)
    written = torch.zeros(s["k"].shape[0], 16, dtype=torch.bool)
    for i, n in enumerate((30, 400)):
        pg, row = P.slots_of(s["table"], i, n, 16, s["k"].shape[0])
        written[pg, row] = True
    written = written.cuda()[:, None, :].expand(-1, 2, -1)
    for x, y in ((one.k, three.k), (one.v, three.v)):
        assert torch.equal(x.isnan(), y.isnan()) and not x[written].isnan().any() and near(x[written], y[written])
        assert x[~written].isnan().all()
    assert torch.equal(one.v[written], three.v[written])
    assert torch.equal(one.position, three.position) and torch.equal(one.weight, three.weight)
