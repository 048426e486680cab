"""More of what the paged cache's entry points refuse: on the CPU calls that are refused, on the GPU such that are taken."""

import random

import pytest
import torch

from paper_2606_22327_amd import kvcache as C
from paper_2606_22327_amd import svfsim as S
from test_kvcache_refusals import A, append, attend, batch, cache


def refused(call, *args):
    assert call(*args, None) == -1
    return C.last_error()


# q and out as offsets, strides and sizes in elements: two tensors of [tokens, heads, 128], and whether they are apart
PLACES = [
    (dict(q=0, out=0), False),                                          # in place
    (dict(q=0, out=2048), True), (dict(q=2048, out=0), True),           # one behind the other
    (dict(q=0, out=2040), False), (dict(q=0, out=1024), False),
    (dict(q=0, out=1024, qt=2048, ot=2048), True),                      # the halves of each token of one buffer
    (dict(q=1024, out=0, qt=2048, ot=2048), True), (dict(q=0, out=1016, qt=2048, ot=2048), False),
    (dict(q=0, out=128, qh=256, oh=256, qt=2048, ot=2048), True),       # every other head
    (dict(q=0, out=120, qh=256, oh=256, qt=2048, ot=2048), False),
    (dict(q=0, out=128, qt=128, ot=128, qh=256, oh=256), False),        # heads outside, tokens inside
    (dict(q=0, out=256, qt=128, ot=128, qh=512, oh=512), True),
    (dict(q=0, out=1024, tokens=1, qt=8, ot=4096), True),               # one token: its stride does not count
    (dict(q=0, out=1024, qt=2048, ot=1024), False),                     # strides that differ: by their ranges
]


def place(q, out, tokens=2, qt=1024, qh=128, ot=1024, oh=128):
    return dict(q=A + 2 * q, out=A + 2 * out, qt=qt, qh=qh, ot=ot, oh=oh), tokens


@pytest.mark.parametrize("kw", [x for x, apart in PLACES if not apart])
def test_attend_refuses_out_over_q(kw):
    at, tokens = place(**kw)
    assert "apart" in refused(S.load().svf_kv_attend, cache(), batch(num_tokens=tokens), attend(**at))


def test_append_refuses_q_out_over_a_part_of_q():
    for off in (8, 1024, 2040):
        assert "apart" in refused(S.load().svf_kv_append, cache(), batch(), append(q_out=A + 2 * off))


def views(q, out, tokens=2, qt=1024, qh=128, ot=1024, oh=128, heads=8, dim=128):
    buf = torch.randn(20000, device="cuda").to(torch.bfloat16)
    return (buf.as_strided((tokens, heads, dim), (qt, qh, 1), q), buf.as_strided((tokens, heads, dim), (ot, oh, 1), out))


def taken(q, out):
    """Whether attend and append take these; what they take has to be right."""
    tokens, heads, dim = q.shape
    ints = dict(dtype=torch.int32, device="cuda")
    k = torch.randn((4, 2, 16, dim), device="cuda").to(torch.bfloat16)
    b = C.Batch(torch.tensor([0, tokens], **ints), torch.tensor([40], **ints), torch.tensor([[2, 0, 1]], **ints), tokens)
    want = C.attend(q.clone(), b, C.Cache(k, k))[0]
    held = q.clone()
    same = out.data_ptr() == q.data_ptr() and out.stride() == q.stride()
    try:
        C.attend(q, b, C.Cache(k, k), out=out)
    except S.SvfError as e:
        assert "apart" in str(e)
        if not same:
            with pytest.raises(S.SvfError):
                C.append(q, k[:tokens, :, 0], k[:tokens, :, 0], torch.zeros(tokens, **ints), None, b, C.Cache(k, k), q_out=out)
        return False
    assert torch.equal(out, want) and torch.equal(q, held)
    C.append(q, k[:tokens, :, 0], k[:tokens, :, 0], torch.zeros(tokens, **ints), None, b, C.Cache(k, k), q_out=out)
    assert torch.equal(out, held)
    return True


@pytest.mark.gpu
@pytest.mark.parametrize("kw,apart", PLACES)
def test_outputs_beside_queries_in_one_buffer(kw, apart):
    assert taken(*views(**kw)) == apart


@pytest.mark.gpu
def test_outputs_and_queries_of_random_strides_against_every_element():
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    for _ in range(200):
        tokens, heads = rng.randint(1, 4), rng.choice((2, 4))
        token_outer = rng.random() < 0.5
        n = heads if token_outer else tokens
        si = 64 * rng.randint(1, 3)
        so = si * (n - 1) + 64 + 64 * rng.randint(0, 2)
        ts, hs = (so, si) if token_outer else (si, so)
        q, out = rng.randrange(0, 2000, 8), rng.randrange(0, 2000, 8)
        rows = lambda at: {at + t * ts + h * hs + d for t in range(tokens) for h in range(heads) for d in range(64)}  # noqa: E731
        apart = not (rows(q) & rows(out))
        assert taken(*views(q, out, tokens, ts, hs, ts, hs, heads, 64)) == apart, (tokens, heads, ts, hs, q, out)
        seen[apart] += 1
    assert min(seen.values()) > 20, seen


def test_launches_of_too_many_threads_are_refused():
    """Sizes within the limits of their numbers whose launch would have 2^32 threads."""
    from test_kvcache_refusals import evict
    lib, many = S.load(), 1 << 26
    for kw in (dict(), dict(qt=1025)):                  # 16 bytes a lane, and element by element
        assert "too large" in refused(lib.svf_kv_append, cache(kv_heads=1), batch(num_tokens=many),
                                      append(heads=1, q_out=A + (1 << 60), **kw))
    big = batch(num_seqs=1 << 21)
    assert "too large" in refused(lib.svf_kv_evict, cache(page_size=4096), big, evict(workspace_bytes=1 << 62))
    seqs = batch(num_seqs=1 << 24, num_tokens=1 << 28, max_q=100)
    assert lib.svf_kv_attend_workspace(cache(), seqs, attend(heads=2)) == -1 and "too large" in C.last_error()
    assert "too large" in refused(lib.svf_kv_attend, cache(), seqs, attend(heads=2, out=A + (1 << 60), workspace_bytes=1 << 62))
    # one less is within the limits, as far as the workspace goes
    assert lib.svf_kv_attend_workspace(cache(), batch(num_seqs=1 << 20, num_tokens=1 << 20, max_q=100), attend(heads=2)) > 0


def host_call(name, grad):
    """A call with host tensors of which ``grad`` requires a gradient; refused either way, by this check or by the next."""
    x = {n: torch.zeros(shape, dtype=torch.bfloat16) for n, shape in
         (("q", (1, 8, 128)), ("k", (1, 2, 128)), ("v", (1, 2, 128)), ("out", (1, 8, 128)), ("keys", (4, 2, 16, 128)),
          ("values", (4, 2, 16, 128)))}
    x["weight"], x["rope"] = torch.zeros((4, 2, 16)), torch.zeros((9, 128))
    if grad:
        x[grad].requires_grad_()
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    b = C.Batch(ints(0, 1), ints(5), ints(0)[None], 1)
    held = C.Cache(x["keys"], x["values"], x["weight"], torch.zeros((4, 2, 16), dtype=torch.int32))
    with pytest.raises(S.SvfError) as e:
        if name == "append":
            C.append(x["q"], x["k"], x["v"], ints(4), x["rope"], b, held, q_out=x["out"])
        elif name == "attend":
            C.attend(x["q"], b, held, add_weight=True, out=x["out"])
        else:
            C.evict(b, held, 4, 1, ints(5))
    assert e.value.name == "SVF_EINVAL"
    return "backward" in str(e.value)


@pytest.mark.parametrize("name,tensors", [("append", ("q", "k", "v", "rope", "keys", "values", "out")),
                                          ("attend", ("q", "keys", "values", "weight", "out")),
                                          ("evict", ("keys", "values", "weight"))])
def test_gradients_are_refused_where_they_would_be_lost(name, tensors):
    for x in tensors:
        assert host_call(name, x), x
        with torch.no_grad():
            assert not host_call(name, x), x
    assert not host_call(name, None)


@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), 1e300, 3e38])
def test_scales_that_are_not_finite_in_32_bits_are_refused(scale):
    assert "scale" in refused(S.load().svf_kv_attend, cache(), batch(), attend(scale=scale))


@pytest.mark.gpu
def test_numbers_past_32_bits_are_refused_as_arguments():
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.zeros((4, 2, 16, 128), dtype=torch.bfloat16, device="cuda")
    held = C.Cache(k, k.clone(), torch.zeros((4, 2, 16), device="cuda"), torch.zeros((4, 2, 16), dtype=torch.int32, device="cuda"))
    b, q = C.Batch(ints(0, 1), ints(20), ints(0, 1)[None], 1), torch.zeros((1, 8, 128), dtype=torch.bfloat16, device="cuda")
    calls = [lambda: C.attend(q, b, held, window=2 ** 31), lambda: C.attend(q, b._replace(max_q=2 ** 40), held),
             lambda: C.attend(q, b._replace(max_q=1.5), held), lambda: C.attend(q, b, held, scale=1e300),
             lambda: C.evict(b, held, 2 ** 31, 0, ints(20)), lambda: C.evict(b, held, 10, -2 ** 31 - 1, ints(20)),
             lambda: C.append(q, k[:1, :, 0], k[:1, :, 0], ints(0), None, b._replace(max_q=2 ** 40), held)]
    for call in calls:
        with pytest.raises(S.SvfError) as e:
            call()
        assert e.value.name == "SVF_EINVAL"
    C.attend(q, b, held, window=2 ** 31 - 1)


@pytest.mark.gpu
def test_an_error_that_another_call_has_left_is_not_these_calls():
    import ctypes
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    k = torch.randn((4, 2, 16, 128), device="cuda").to(torch.bfloat16)
    held = C.Cache(k, k.clone(), torch.zeros((4, 2, 16), device="cuda"), torch.zeros((4, 2, 16), dtype=torch.int32, device="cuda"))
    b, q = C.Batch(ints(0, 1), ints(20), ints(0, 1)[None], 1), torch.randn((1, 8, 128), device="cuda").to(torch.bfloat16)
    many = C.Batch(ints(0, 20), ints(20), ints(0, 1)[None], 20)
    qs, new = q.expand(20, 8, 128).contiguous(), ints(20)
    hip = S.load()
    hip.hipSetDevice.argtypes = [ctypes.c_int]
    for call in (lambda: C.attend(q, b, held, add_weight=True), lambda: C.attend(qs, many, held, add_weight=True),
                 lambda: C.append(q, k[:1, :, 3], k[:1, :, 3], ints(0), None, b, held), lambda: C.evict(b, held, 10, 0, new)):
        call()                                          # torch has what it hands out, and asks for no more
        torch.cuda.synchronize()
        assert hip.hipSetDevice(1 << 20) != 0           # refused; leaves its error for whoever asks
        try:
            call()
        finally:
            hip.hipGetLastError()
