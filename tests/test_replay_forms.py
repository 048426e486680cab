"""Schedules replayed with images, windows and scored answers: the host's part (CPU), and all of it together (GPU)."""

import numpy as np
import pytest

from paper_2606_22327_amd import replay as R
from paper_2606_22327_amd import workloads as W
from test_replay import schedule


def test_grid_positions():
    t = R.TEXT
    p = R.grid_positions(np.arange(2 * (t + 6) + 3), 1000, (2, 3))
    assert p[:t].tolist() == [[i, i, i] for i in range(t)]
    assert p[t:t + 6].tolist() == [[t, t + y, t + x] for y in range(2) for x in range(3)]
    assert p[t + 6].tolist() == [t + 3] * 3                          # behind the larger side
    assert p[2 * t + 6].tolist() == [2 * t + 3] * 3 and p[-1].tolist() == [2 * t + 6 + 2] * 3
    # answers are text, wherever the prompt ended
    for prompt, nxt in ((5, 5), (t, t), (t + 1, t + 3), (t + 6, t + 3), (t + 7, t + 4)):
        a = R.grid_positions(prompt + np.arange(3), prompt, (2, 3))
        assert a.tolist() == [[nxt + i] * 3 for i in range(3)], prompt
        before = R.grid_positions(np.arange(prompt), prompt, (2, 3))
        assert before.max() < nxt


@pytest.mark.parametrize("grid", [(1, 1), (1, 9), (9, 1), (4, 4)])
def test_positions_stay_inside_the_table(grid):
    prompt = np.arange(1, 300)
    token = prompt + 50
    assert (R.grid_positions(token, prompt, grid).max(-1) <= token + max(grid)).all()
    assert (R.grid_positions(np.minimum(np.arange(299), prompt - 1), prompt, grid).max(-1) <= np.arange(299) + max(grid)).all()


def test_pages_given_back_are_handed_out_again_and_once():
    rng = np.random.default_rng(2)
    pages = R.Pages(60, 8)
    length = {}
    for _ in range(500):
        i = int(rng.integers(0, 6))
        n = int(rng.integers(length.get(i, 0), 90)) if rng.random() < 0.8 else 0
        pages.resize(i, n)
        length[i] = n
        if n:
            pages.give_back(i, 5, n + 1 - 20)
        all_ = [p for x in pages.held.values() for p in x if p >= 0]
        assert len(set(all_)) == len(all_) and sorted(all_ + pages.free) == list(range(60))
        for j, held in pages.held.items():
            for at, p in enumerate(held):       # what the next token sees is there
                seen = any(s < 5 or s >= length[j] + 1 - 20 for s in range(at * 8, min(at * 8 + 8, length[j])))
                assert p >= 0 or not seen


def test_keep_and_window_exclude_each_other():
    with pytest.raises(ValueError, match="not both"):
        R.Replay([3], [2], [0], 100, keep=8, window=8)


@pytest.mark.gpu
@pytest.mark.parametrize("window,first,grid,page", [(24, 4, None, 16), (10, 20, (3, 5), 4), (7, 0, (2, 2), 1), (0, 0, (4, 4), 16)])
def test_replayed_steps_against_the_plain_forms(window, first, grid, page):
    import torch
    import kv_plain as P
    from test_kvcache_first import plain
    from test_logprobs import near, plain as plain_scores
    b, got = schedule(1, 14)
    r = R.Replay(b.prompt, b.output, got["start"], b.M, heads=8, kv_heads=2, dim=64, page=page, window=window, first=first,
                 grid=grid, vocab=1000, top=3)
    steps = 0
    while True:
        s = r.step()
        if s is None:
            break
        steps += 1
        assert s["held"] <= b.M
        cache, batch = r.cache, s["batch"]
        state = {"q": s["q"].cpu(), "k": cache.k.cpu(), "v": cache.v.cpu(), "offsets": batch.q_offsets.cpu(),
                 "kv_len": batch.kv_len.cpu(), "table": batch.page_table.cpu()}
        out, lse, _, tol = plain(state, True, window, first, 64 ** -0.5)
        e = P.out_tolerance(s["q"].dtype, 64, out, tol, int(batch.kv_len.max()))
        assert ((s["out"].cpu().double() - out).abs() <= e).all()
        assert ((s["lse"].cpu().double() - lse).abs() <= P.lse_tolerance(64, lse, tol)).all()
        lp, entropy, rank, top_lp, index, t0, t1, t2 = plain_scores(s["logits"].cpu(), s["token"].cpu(), 3, 1.0)
        assert torch.equal(s["score"].rank.cpu().long(), rank) and torch.equal(s["score"].top_index.cpu().long(), index)
        near(s["score"].logprob, lp, t0)
        near(s["score"].entropy, entropy, t2)
    assert steps >= int(b.output.max()) and not r.pages.held and len(r.pages.free) == r.cache.k.shape[0]


@pytest.mark.gpu
def test_a_window_over_everything_reads_what_no_window_does():
    import torch
    b, got = schedule(1, 10)
    a, c = (R.Replay(b.prompt, b.output, got["start"], b.M, heads=4, kv_heads=2, dim=64, window=w, first=4, grid=(2, 3))
            for w in (0, 100000))
    while True:
        x, y = a.step(), c.step()
        if x is None:
            break
        assert torch.equal(x["out"], y["out"]) and torch.equal(x["lse"], y["lse"]) and x["held"] == y["held"] and x["read"] == y["read"]
    assert y is None


@pytest.mark.gpu
def test_images_shrunk_by_weight_keep_the_order_of_the_text():
    b, got = schedule(1, 14)
    r = R.Replay(b.prompt, b.output, got["start"], b.M, heads=4, kv_heads=2, dim=64, keep=24, grid=(4, 4))
    steps = 0
    while True:
        s = r.step()
        if s is None:
            break
        steps += 1
        # what the cache keeps of a request that it has shrunk: the first 4 tokens, and the newest of the text
        batch, pos = s["batch"], r.cache.position.cpu()
        for i, (n, request) in enumerate(zip(batch.kv_len.tolist(), s["request"])):
            if n > 24 and int(request) in r.pages.held:
                pages = r.pages.held[int(request)]
                kept = [int(pos[pages[j // 16], 0, j % 16]) for j in range(24)]
                newest = int(r.prompt[request]) + int(s["time"] - got["start"][request])
                assert len(set(kept)) == 24 and set(range(4)) <= set(kept) and set(range(newest - 5, newest + 1)) <= set(kept)
    assert steps > 0


@pytest.mark.gpu
def test_replay_of_a_workload_with_a_window_and_scores():
    sums = R.run(W.config(2, instances=1, n=30), heads=8, kv_heads=2, dim=64, window=64, first=4, grid=(8, 8), vocab=5000, top=2)
    whole = R.run(W.config(2, instances=1, n=30), heads=8, kv_heads=2, dim=64)
    assert sums["slots_read"] < whole["slots_read"] and sums["most_slots"] < whole["most_slots"] and sums["steps"] == whole["steps"] and sums["tokens"] == whole["tokens"]
    # random tokens among 5,000 with logits of variance 9: ln 5000 + 4.5 each
    tokens = int(W.config(2, instances=1, n=30).output.sum())
    assert 0.8 < sums["nats"] / (tokens * (np.log(5000) + 4.5)) < 1.2
