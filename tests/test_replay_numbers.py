"""Every call that a replayed schedule makes of the cache, against the plain forms in 64 bits: what append writes, what attention returns and
adds to the weights, what eviction moves, step after step on the state that the steps before have left."""

import numpy as np
import pytest
import torch

import kv_plain as P
import oracle
from paper_2606_22327_amd import replay as R
from paper_2606_22327_amd import workloads as W

pytestmark = pytest.mark.gpu


def on_cpu(cache):
    return [x.cpu() for x in cache]


class Checked:
    """The cache's calls, each compared with its plain form."""

    def __init__(self, module, monkeypatch):
        self.calls = {"append": 0, "attend": 0, "evict": 0}
        self.moved = 0
        for name in self.calls:
            monkeypatch.setattr(module, name, lambda *a, _f=getattr(module, name), _n=name, **kw: getattr(self, _n)(_f, *a, **kw))

    def append(self, f, q, k, v, positions, rope, batch, cache):
        before = [None if x is None else x.cpu() for x in cache]
        q0, k0, v0, pos = q.cpu(), k.cpu(), v.cpu(), positions.cpu()
        got = f(q, k, v, positions, rope, batch, cache)
        cos, sin = rope.cpu()[pos.long()].double().chunk(2, 1)
        want_q, want_k = (P.rotate(x.double(), cos, sin, "half") for x in (q0, k0))
        kp, vp, wp, pp = before[0].double(), before[1], before[2], before[3]
        page = kp.shape[2]
        for i, n in enumerate(batch.kv_len.tolist()):
            a, b = batch.q_offsets[i].item(), batch.q_offsets[i + 1].item()
            pg, row = (x[n - (b - a):] for x in P.slots_of(batch.page_table.cpu(), i, n, page, kp.shape[0]))
            kp[pg, :, row], vp[pg, :, row] = want_k[a:b], v0[a:b]
            if wp is not None:
                wp[pg, :, row], pp[pg, :, row] = 0.0, pos[a:b, None]
        u, size = P.UNIT[q.dtype], q0.double().abs().max()

        def near(x, y):         # what no slot has held may be anything
            x, ok = x.cpu().double(), y.isfinite()
            assert ((x - y).abs() <= u * y.abs() * 1.01 + 2.0 ** -22 * size + 2.0 ** -25)[ok].all()

        near(got, want_q)
        near(cache.k, kp)
        assert torch.equal(torch.nan_to_num(cache.v.cpu()), torch.nan_to_num(vp))
        assert wp is None or (torch.equal(cache.weight.cpu(), wp) and torch.equal(cache.position.cpu(), pp))
        self.calls["append"] += 1
        return got

    def attend(self, f, q, batch, cache, add_weight=False):
        before = None if cache.weight is None else cache.weight.cpu().double()
        out, lse = f(q, batch, cache, add_weight=add_weight)
        D = q.shape[2]
        lens = batch.kv_len.cpu()
        want, want_lse, add, tol = P.attend(q.cpu(), cache.k.cpu(), cache.v.cpu(), batch.q_offsets.cpu(), lens, batch.page_table.cpu(),
                                            True, 0, D ** -0.5)
        assert ((out.cpu().double() - want).abs() <= P.out_tolerance(q.dtype, D, want, tol, int(lens.max()))).all()
        assert ((lse.cpu().double() - want_lse).abs() <= P.lse_tolerance(D, want_lse, tol)).all()
        if add_weight:
            rows = batch.max_q * q.shape[1] // cache.k.shape[1]
            z = cache.weight.cpu().double() - before
            assert ((z - add).abs() <= P.weight_tolerance(D, before, add, tol, rows)).all()
        self.calls["attend"] += 1
        return out, lse

    def evict(self, f, batch, cache, budget, recent, first, next_position):
        before = on_cpu(cache)
        got = f(batch, cache, budget, recent=recent, first=first, next_position=next_position)
        want = P.evict(*before, batch.kv_len.cpu(), batch.page_table.cpu(), budget, recent, first, next_position.cpu())
        assert torch.equal(got.cpu(), want[4])
        for x, y in zip(cache, want):
            assert torch.equal(torch.nan_to_num(x.cpu()), torch.nan_to_num(y))
        self.calls["evict"] += 1
        self.moved += int((before[3] != want[3]).sum())
        return got


@pytest.mark.parametrize("keep,steps", [(None, 12), (24, 40), (9, 12)])
def test_every_call_of_a_replay_against_its_plain_form(keep, steps, monkeypatch):
    b = W.config(1, instances=1, n=14).subset([0])
    r = R.Replay(b.prompt, b.output, oracle.run(b, "svf")["start"], b.M, heads=8, kv_heads=2, dim=64, page=16, keep=keep)
    seen = Checked(r.C, monkeypatch)
    done = 0
    while done < steps and r.step() is not None:
        done += 1
        held = r.length[r.length > 0]
        assert held.sum() <= b.M and (keep is None or np.all(held <= keep))
    assert done > 8 and seen.calls["append"] == seen.calls["attend"] == done and seen.calls["evict"] == (done if keep else 0)
    assert keep is None or seen.moved > 0
