"""Schedules replayed on the paged cache: what the host plans (CPU) and what the kernels compute (GPU)."""

import numpy as np
import pytest

import oracle
from paper_2606_22327_amd import replay as R
from paper_2606_22327_amd import workloads as W


def schedule(cfg, n, instance=0):
    b = W.config(cfg, instances=instance + 1, n=n).subset([instance])
    return b, oracle.run(b, "svf")


@pytest.mark.parametrize("cfg,n", [(1, 50), (2, 40), (4, 12)])
def test_timeline_holds_what_the_memory_model_counts(cfg, n):
    b, got = schedule(cfg, n)
    s, o, k = b.prompt.astype(np.int64), b.output.astype(np.int64), got["start"].astype(np.int64)
    read, steps = 0, np.zeros(len(s), dtype=np.int64)
    for step in R.timeline(s, o, k):
        tau = step.time + 1
        held = (step.age + step.new)
        assert np.array_equal(held, s[step.request] + tau - k[step.request])      # eq:c2
        assert held.sum() <= b.M
        read += held.sum()
        steps[step.request] += 1
    assert np.array_equal(steps, o)
    assert read == (s * o + (o * o + o) // 2).sum()                                # Eq. 1


def test_timeline_skips_idle_steps():
    t = [(x.time, x.request.tolist(), x.new.tolist(), x.age.tolist()) for x in R.timeline([3, 2], [2, 1], [0, 10])]
    assert t == [(0, [0], [4], [0]), (1, [0], [1], [4]), (10, [1], [3], [0])]
    assert list(R.timeline([], [], [])) == []


def test_pages_are_handed_out_once():
    rng = np.random.default_rng(1)
    pages = R.Pages(40, 16)
    for _ in range(300):
        i, n = int(rng.integers(0, 8)), int(rng.integers(0, 70))
        pages.resize(i, n)
        all_ = [p for x in pages.held.values() for p in x]
        assert len(set(all_)) == len(all_) and sorted(all_ + pages.free) == list(range(40))
        assert len(pages.held.get(i, [])) == -(-n // 16)
    pages.resize(3, 33)
    pages.resize(4, 1)
    t = pages.table([3, 4])
    assert t.shape == (2, 3) and t[0].tolist() == pages.held[3] and t[1, 0] == pages.held[4][0]


@pytest.mark.gpu
@pytest.mark.parametrize("keep", [None, 24])
def test_replayed_steps_against_the_plain_attention(keep):
    import kv_plain as P
    b, got = schedule(1, 14)
    r = R.Replay(b.prompt, b.output, got["start"], b.M, heads=8, kv_heads=2, dim=64, page=16, keep=keep)
    steps = 0
    while True:
        s = r.step()
        if s is None:
            break
        steps += 1
        assert s["held"] <= b.M
        if keep:
            assert s["held"] <= keep * len(s["request"])
            continue                # the cache has moved on: eviction came after attention
        cache, batch = r.cache, s["batch"]
        out, lse, _, tol = P.attend(s["q"].cpu(), cache.k.cpu(), cache.v.cpu(), batch.q_offsets.cpu(), batch.kv_len.cpu(),
                                    batch.page_table.cpu(), True, 0, 64 ** -0.5)
        e = P.out_tolerance(s["q"].dtype, 64, out, tol, int(batch.kv_len.max()))
        assert ((s["out"].cpu().double() - out).abs() <= e).all()
        assert ((s["lse"].cpu().double() - lse).abs() <= P.lse_tolerance(64, lse, tol)).all()
    assert steps >= int(b.output.max()) and not r.pages.held and len(r.pages.free) == r.cache.k.shape[0]


@pytest.mark.gpu
def test_replay_of_a_workload():
    sums = R.run(W.config(1, instances=1), heads=8, kv_heads=2, dim=64)
    assert sums["slots_read"] == sums["volume"] and sums["most_slots"] <= sums["M"] == 512 and sums["requests"] == 50
    less = R.run(W.config(2, instances=1, n=30), keep=64, heads=8, kv_heads=2, dim=64)
    assert less["slots_read"] < less["volume"]
