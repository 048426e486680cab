"""The calls have no derivatives and no place in a trace: what would be lost without a word is refused."""

import pytest
import torch
import torch.autograd.forward_ad as fw

from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import logprobs as L
from paper_2606_22327_amd import svfsim as S

BF = torch.bfloat16


def calls(dev):
    """name -> (function of some tensors, the tensors, which of them may have a derivative)"""
    g = torch.Generator().manual_seed(1)

    def r(*shape, dtype=BF):
        return torch.randn(shape, generator=g).to(dtype).to(dev)

    def whole(*x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    k, v, weight, position = r(4, 2, 16, 64), r(4, 2, 16, 64), torch.zeros((4, 2, 16), device=dev), torch.zeros((4, 2, 16), dtype=torch.int32, device=dev)
    batch = C.Batch(whole(0, 1, 2), whole(20, 3), whole(0, 1, 2, 3).view(2, 2), 1)
    q, kn, vn, rope = r(2, 4, 64), r(2, 2, 64), r(2, 2, 64), torch.rand((30, 64), generator=g).to(dev)
    pos, axes = whole(5, 9), C.pair_axes((16, 16))
    x, token = r(2, 50, dtype=torch.float32), whole(3, 4).long()
    return {
        "append": (lambda q, kn, vn, k, v, rope: C.append(q, kn, vn, pos, rope, batch, C.Cache(k, v)), (q, kn, vn, k, v, rope)),
        "axes": (lambda q, kn, vn, k, v, rope: C.append(q, kn, vn, pos[:, None].expand(2, 2), rope, batch, C.Cache(k, v), axes=axes),
                 (q, kn, vn, k, v, rope)),
        "q_out": (lambda out: C.append(q, kn, vn, pos, rope, batch, C.Cache(k, v), q_out=out), (torch.empty_like(q),)),
        "attend": (lambda q, k, v, weight: C.attend(q, batch, C.Cache(k, v, weight), add_weight=True)[0], (q, k, v, weight)),
        "first": (lambda q, k, v: C.attend(q, batch, C.Cache(k, v), window=4, first=2)[0], (q, k, v)),
        "out": (lambda out: C.attend(q, batch, C.Cache(k, v), out=out)[0], (torch.empty_like(q),)),
        "evict": (lambda k, v, weight: C.evict(batch, C.Cache(k, v, weight, position), 8, 2, whole(20, 3)), (k, v, weight)),
        "score": (lambda x: L.score(x, token).logprob, (x,)),
    }


NAMES = ("append", "axes", "q_out", "attend", "first", "out", "evict", "score")


def duals_are_refused(name, dev):
    f, tensors = calls(dev)[name]
    for i, t in enumerate(tensors):
        with fw.dual_level():
            dual = fw.make_dual(t, torch.ones_like(t))
            with pytest.raises(S.SvfError, match="forward mode"):
                f(*tensors[:i], dual, *tensors[i + 1:])


def traces_are_refused(name, dev):
    from torch.fx.experimental.proxy_tensor import make_fx
    f, tensors = calls(dev)[name]
    with pytest.raises(S.SvfError, match="traced"):
        torch.jit.trace(f, tensors, check_trace=False)
    with pytest.raises(S.SvfError, match="traced"):
        make_fx(f)(*tensors)


@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused(name):
    duals_are_refused(name, "cpu")


@pytest.mark.parametrize("name", NAMES)
def test_traces_are_refused(name):
    traces_are_refused(name, "cpu")


@pytest.mark.parametrize("name", NAMES)
def test_gradients_are_refused(name):
    f, tensors = calls("cpu")[name]
    for i, t in enumerate(tensors):
        with pytest.raises(S.SvfError, match="backward"):
            f(*tensors[:i], t.clone().requires_grad_(), *tensors[i + 1:])


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_the_binding_takes_none_of_them(name):
    duals_are_refused(name, "cuda")
    traces_are_refused(name, "cuda")
    f, tensors = calls("cuda")[name]
    want = f(*(t.clone() for t in tensors))
    with fw.dual_level():           # a level without duals, and a mode that only looks on, change nothing
        assert torch.equal(f(*(t.clone() for t in tensors)), want)
    from torch.utils.flop_counter import FlopCounterMode
    with FlopCounterMode(display=False):
        assert torch.equal(f(*(t.clone() for t in tensors)), want)
    for t in tensors:
        t.requires_grad_()
    with torch.no_grad():
        assert torch.equal(f(*tensors), want)
