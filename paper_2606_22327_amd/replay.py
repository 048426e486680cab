"""Replays a simulated schedule on one layer's paged key-value cache.

    python -m paper_2606_22327_amd.replay [--config 1] [--instance 0] [--requests N] [--policy svf]
                                          [--keep SLOTS | --window SLOTS [--first SLOTS]] [--grid H W]
                                          [--vocab V [--top K]] [--heads 32] [--kv-heads 8] [--dim 128] [--page 16]

The simulator plans with a budget of M cache slots and steps of one token for
every running request.  Here each simulated step is carried out: the running
requests' new tokens are appended to their pages and attend to everything that
their request holds.  A request's first step brings its prompt and its first
token (s + 1 slots, what the memory model counts after the start step), every later one a
token; at its finish its pages go back.  The slots that attention reads over
a run are then, exactly, the sum of the requests' volumes (Eq. 1), and the slots held
after a step never exceed M.

``--keep`` is the other way to live with little memory than evicting whole requests:
each request is held to that many slots, those of the largest attention weight, the
first 4 tokens and the newest quarter.  ``--window`` is a third: a token sees so many slots up to its own and the request's
``--first`` slots, and the pages that no token will see again go back.

``--grid`` makes prompts of texts and images of H x W tokens, whose positions have three axes.  ``--vocab`` ends
a step with the log probability of each request's token among so many, and the ``--top`` best.

Queries, keys, values and logits are random numbers in place of a model's projections.
"""

from __future__ import annotations

import argparse
import json
from typing import Dict, Iterator, List, NamedTuple, Optional, Tuple

import numpy as np


class Step(NamedTuple):
    """One simulated step: for each running request its number, new tokens and age (tokens before them)."""

    time: int
    request: np.ndarray
    new: np.ndarray
    age: np.ndarray


def timeline(prompt, output, start) -> Iterator[Step]:
    """The steps of a schedule in which something runs: request i from start[i] on, for
    output[i] steps (it must have started and not have been evicted)."""
    prompt, output, start = (np.asarray(x, dtype=np.int64) for x in (prompt, output, start))
    order = np.argsort(start, kind="stable")
    running: List[int] = []
    at, t, n = 0, 0, len(order)
    while at < n or running:
        if not running:
            t = int(start[order[at]])
        while at < n and start[order[at]] == t:
            running.append(int(order[at]))
            at += 1
        r = np.array(running, dtype=np.int64)
        x = t - start[r]                                   # tokens generated before this step
        yield Step(t, r, np.where(x == 0, prompt[r] + 1, 1), np.where(x == 0, 0, prompt[r] + x))
        t += 1
        running = [i for i in running if t - start[i] < output[i]]


#: Tokens of text before each image of a prompt with a grid.
TEXT = 32


def grid_positions(token, prompt, grid: Tuple[int, int]) -> np.ndarray:
    """Time, row and column of tokens (their numbers in requests of ``prompt`` tokens): in a prompt ``TEXT`` tokens of
    text and an image of grid[0] x grid[1] tokens follow each other.  Text counts on every axis; in an image time
    stands still, rows and columns count from there, and what follows goes on behind the larger of the two.  Answers are text."""
    token, prompt = np.asarray(token, dtype=np.int64), np.asarray(prompt, dtype=np.int64)
    h, w = grid
    at = np.minimum(token, prompt)                       # an answer counts on from the prompt's end
    turn, i = at // (TEXT + h * w), at % (TEXT + h * w)
    start = turn * (TEXT + max(h, w)) + np.minimum(i, TEXT)
    inside = np.maximum(i - TEXT, 0)
    answer = token >= prompt
    start = start + np.where(answer, token - prompt + np.where(i > TEXT, max(h, w), 0), 0)
    inside = np.where(answer, 0, inside)
    return np.stack((start, start + inside // w, start + inside % w), -1)


class Pages:
    """Page lists of the running requests out of one pool; -1 where a page was given back."""

    def __init__(self, num_pages: int, page: int):
        self.page = page
        self.free = list(range(num_pages - 1, -1, -1))
        self.held: Dict[int, List[int]] = {}

    def resize(self, request: int, slots: int):
        """The request holds ``slots`` slots from now on (0: it is gone)."""
        pages = self.held.setdefault(request, [])
        need = -(-slots // self.page)
        while len(pages) < need:
            pages.append(self.free.pop())
        while len(pages) > need:
            last = pages.pop()
            if last >= 0:
                self.free.append(last)
        if not pages:
            del self.held[request]

    def give_back(self, request: int, begin: int, end: int):
        """The request holds none of the slots [begin, end) any more: pages that hold nothing else go back."""
        pages = self.held[request]
        for i in range(-(-begin // self.page), min(end // self.page, len(pages))):
            if pages[i] >= 0:
                self.free.append(pages[i])
                pages[i] = -1

    def table(self, requests) -> np.ndarray:
        lists = [self.held[int(i)] for i in requests]
        out = np.zeros((len(lists), max(map(len, lists))), dtype=np.int32)
        for row, pages in zip(out, lists):
            row[: len(pages)] = pages
        return out


class Replay:
    """A schedule's requests on one layer's cache, step by step.

    ``M`` is the budget in slots; the pool has as many, and for each request that runs
    a page more, which is what pages that are not full can cost."""

    def __init__(self, prompt, output, start, M: int, heads: int = 32, kv_heads: int = 8, dim: int = 128,
                 page: int = 16, keep: Optional[int] = None, seed: int = 0, window: int = 0, first: int = 0,
                 grid: Optional[Tuple[int, int]] = None, vocab: int = 0, top: int = 0):
        import torch
        from . import kvcache, logprobs

        if keep and window:
            raise ValueError("a window counts slots, which eviction moves: keep or window, not both")
        self.torch, self.C, self.L = torch, kvcache, logprobs
        self.window, self.first, self.grid, self.vocab, self.top = window, first, grid, vocab, top
        self.steps = timeline(prompt, output, start)
        self.prompt, self.output = np.asarray(prompt, dtype=np.int64), np.asarray(output, dtype=np.int64)
        self.M, self.heads, self.kv_heads, self.dim, self.keep = int(M), heads, kv_heads, dim, keep
        most = max((len(s.request) for s in timeline(prompt, output, start)), default=0)
        num_pages = -(-self.M // page) + most
        self.pages = Pages(num_pages, page)
        self.length = np.zeros(len(self.prompt), dtype=np.int64)     # slots of each request
        pool = (num_pages, kv_heads, page)
        gpu = dict(device="cuda")
        self.cache = kvcache.Cache(torch.empty((*pool, dim), dtype=torch.bfloat16, **gpu),
                                   torch.empty((*pool, dim), dtype=torch.bfloat16, **gpu),
                                   torch.zeros(pool, **gpu) if keep else None,
                                   torch.zeros(pool, dtype=torch.int32, **gpu) if keep else None)
        # an image of one row or column is the largest step of a position
        far = int((self.prompt + self.output).max(initial=0)) + 1 + (max(grid) if grid else 0)
        self.rope = kvcache.rope_table(far, dim)
        self.axes = kvcache.pair_axes((dim // 2 - 2 * (dim // 6), dim // 6, dim // 6)) if grid else None
        self.random = torch.Generator(device="cuda").manual_seed(seed)

    def step(self):
        """Carries out the next step; what it did, or None at the end of the schedule."""
        torch, C = self.torch, self.C
        s = next(self.steps, None)
        if s is None:
            return None
        length = self.length[s.request] + s.new
        for i, n in zip(s.request, length):
            self.pages.resize(int(i), int(n))
        offsets = np.concatenate(([0], np.cumsum(s.new)))
        tokens = int(offsets[-1])
        owner = np.repeat(np.arange(len(s.request)), s.new)
        position = s.age[owner] + np.arange(tokens) - offsets[owner]
        gpu = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()  # noqa: E731
        batch = C.Batch(gpu(offsets), gpu(length), gpu(self.pages.table(s.request)), int(s.new.max()))
        qkv = torch.randn((tokens, self.heads + 2 * self.kv_heads, self.dim), dtype=torch.bfloat16, device="cuda",
                          generator=self.random)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
        if self.grid:
            places = grid_positions(position, self.prompt[s.request][owner], self.grid)
            q = C.append(q, k, v, gpu(places), self.rope, batch, self.cache, axes=self.axes, kept=gpu(position))
        else:
            q = C.append(q, k, v, gpu(position), self.rope, batch, self.cache)
        if self.window:
            out, lse = C.attend(q, batch, self.cache, window=self.window, first=self.first)
        else:
            out, lse = C.attend(q, batch, self.cache, add_weight=bool(self.keep))
        read = length
        if self.window:                     # what the oldest new token's window hides from all, but for the first tokens
            hidden = np.maximum(length - s.new - self.window + 1, 0)
            read = length - hidden + np.minimum(self.first, hidden)
        score = None
        if self.vocab:
            requests = len(s.request)
            logits = 3 * torch.randn((requests, self.vocab), dtype=torch.bfloat16, device="cuda", generator=self.random)
            token = torch.randint(self.vocab, (requests,), device="cuda", generator=self.random)
            score = self.L.score(logits, token, top=self.top)
        if self.keep:
            C.evict(batch, self.cache, self.keep, recent=self.keep // 4, first=min(4, self.keep // 2),
                    next_position=gpu(s.age + s.new))
            length = np.minimum(length, self.keep)
        done = s.time + 1 - self._start(s) >= self.output[s.request]
        self.length[s.request] = np.where(done, 0, length)
        for i, n in zip(s.request, self.length[s.request]):
            self.pages.resize(int(i), int(n))
            if self.window and n:       # the next token's window begins at slot n + 1 - window
                self.pages.give_back(int(i), self.first, int(n) + 1 - self.window)
        held = length
        if self.window:
            hidden = np.maximum(length + 1 - self.window, 0)
            held = length - hidden + np.minimum(self.first, hidden)
        result = {"time": s.time, "request": s.request, "batch": batch, "q": q, "out": out, "lse": lse,
                  "read": int(read.sum()), "tokens": tokens, "held": int(held.sum())}
        if score is not None:
            result.update(logits=logits, token=token, score=score)
        return result

    def _start(self, s: Step) -> np.ndarray:
        age = s.age - self.prompt[s.request]                 # tokens generated before the step
        return s.time - np.where(s.age == 0, 0, age)


def run(batch, policy: str = "svf", instance: int = 0, **kw) -> Dict[str, float]:
    """Simulates one instance of a ``workloads`` batch and replays it; sums over the run."""
    import torch
    from . import svfsim

    one = batch.subset([instance])
    with svfsim.Simulator.from_batch(one, policies=[policy]) as sim:
        sim.run()
        got = sim.read(0)
    if (got["preempt"] > 0).any() or (got["finish"] < 0).any():
        raise ValueError("only schedules that finish without evictions are replayed")
    r = Replay(one.prompt, one.output, got["start"], one.M, **kw)
    sums = {"steps": 0, "tokens": 0, "slots_read": 0, "most_slots": 0}
    nats = torch.zeros((), dtype=torch.float64, device="cuda")
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    while True:
        s = r.step()
        if s is None:
            break
        sums["steps"] += 1
        sums["tokens"] += s["tokens"]
        sums["slots_read"] += s["read"]
        sums["most_slots"] = max(sums["most_slots"], s["held"])
        if r.vocab:
            nats -= s["score"].logprob.sum()
    b.record()
    torch.cuda.synchronize()
    if r.vocab:
        sums["nats"] = round(float(nats), 1)
    o, p = one.output.astype(np.int64), one.prompt.astype(np.int64)
    sums.update(requests=len(o), M=int(one.M), volume=int((p * o + (o * o + o) // 2).sum()),
                us_per_step=round(a.elapsed_time(b) * 1e3 / max(sums["steps"], 1), 1))
    return sums


def main(argv=None):
    from . import workloads

    ap = argparse.ArgumentParser(description="Replay a simulated schedule on one layer's paged cache.")
    ap.add_argument("--config", type=int, default=1, choices=(1, 2, 4))
    ap.add_argument("--instance", type=int, default=0)
    ap.add_argument("--requests", type=int, default=None)
    ap.add_argument("--policy", default="svf", choices=("svf", "sjf", "fcfs"))
    ap.add_argument("--keep", type=int, default=None)
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--first", type=int, default=4)
    ap.add_argument("--grid", type=int, nargs=2, default=None, metavar=("H", "W"))
    ap.add_argument("--vocab", type=int, default=0)
    ap.add_argument("--top", type=int, default=0)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--dim", type=int, default=128)
    ap.add_argument("--page", type=int, default=16)
    a = ap.parse_args(argv)
    batch = workloads.config(a.config, instances=a.instance + 1, n=a.requests)
    print(json.dumps(run(batch, a.policy, a.instance, heads=a.heads, kv_heads=a.kv_heads, dim=a.dim, page=a.page,
                         keep=a.keep, window=a.window, first=a.first, grid=a.grid and tuple(a.grid), vocab=a.vocab,
                         top=a.top)))


if __name__ == "__main__":
    main()
