"""The paged key-value cache behind the simulated budget (``include/svfkv.h``).

A schedule of ``svfsim`` counts cache slots; these calls are what one of its
steps does to a layer's cache on the GPU:

``append``   rotary positions (with one axis or several) on new queries and keys, keys and values into pages
``attend``   attention of new tokens (one or many for each sequence) over the pages: all, a window, or a window and the first tokens
``evict``    shrinks sequences to a number of slots by accumulated attention weight
``rope_table``   cosines and sines by position, for the rotation
``pair_axes``   which axis of a position each pair of a head turns by

Argument marshalling only, in ``csrc/svf_binding.cpp`` for ordinary arguments and here for all others (for all, with a
warning, where that is not built): every step runs in
the HIP kernels of ``libsvfsim.so``, on torch's current stream of the tensors' device.  All tensors are
on one GPU.  There are no derivatives: tensors that require a gradient, where gradients are recorded, and
tensors with a tangent of forward mode are refused, and so is a call that is being traced.  Arguments that can be checked on the host are, and raise
``svfsim.SvfError`` (``SVF_EINVAL``); what lengths, offsets and page numbers in
device memory do is said in ``svfkv.h``.
"""

from __future__ import annotations

import math
import struct
import sys
import warnings
from typing import NamedTuple, Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from . import svfsim

DTYPE = {torch.bfloat16: 0, torch.float16: 1}
LAYOUT = {"half": 0, "interleaved": 1}
MOST_AXES = 4

# the structs of svfkv.h
_CACHE = struct.Struct("@4P6q5i4x")
_BATCH = struct.Struct("@3Pq4i")
_APPEND = struct.Struct("@6P8q4i")
_ATTEND = struct.Struct("@4P5qf4i4x")
_EVICT = struct.Struct("@3Pq3i4x")
_AXES = struct.Struct("@P2qi128s4x")


class Cache(NamedTuple):
    """One layer's pool of pages.  ``k``, ``v``: [num_pages, kv_heads, page_size,
    head_dim], bfloat16 or float16; any strides that are multiples of 8 with
    head_dim contiguous, so a pool kept as [num_pages, page_size, kv_heads,
    head_dim] is passed as its ``transpose(1, 2)``.  ``weight`` (float32) and
    ``position`` (int32): [num_pages, kv_heads, page_size], contiguous, or
    None where a program does not evict."""

    k: torch.Tensor
    v: torch.Tensor
    weight: Optional[torch.Tensor] = None
    position: Optional[torch.Tensor] = None


class Batch(NamedTuple):
    """The sequences of a step (int32 tensors).  ``q_offsets`` [seqs + 1]: new tokens
    q_offsets[i] .. q_offsets[i + 1] - 1 belong to sequence i (None for ``evict``).
    ``kv_len`` [seqs]: slots of each with the new tokens among them, which are
    the last.  ``page_table`` [seqs, pages].  ``max_q``: no sequence has more new
    tokens (the results of one that has are NaN)."""

    q_offsets: Optional[torch.Tensor]
    kv_len: torch.Tensor
    page_table: torch.Tensor
    max_q: int = 1


def _need(ok: bool, text: str):
    if not ok:
        raise svfsim.SvfError(-1, text)


def last_error() -> str:
    return svfsim.load().svf_kv_last_error().decode(errors="replace")


def _check(rc: int, error=last_error):
    if rc != 0:
        raise svfsim.SvfError(rc, error())


# What follows is the long way, for whatever the binding has not taken: another device than the current one, tensors of
# derivatives, traces, arguments to be refused.  The checks are one expression each where all is well; which of them failed is found out afterwards.

def _pack(cache: Cache, batch: Batch, tokens: int) -> Tuple[bytes, bytes]:
    k, v, weight, position = cache
    offsets, kv_len, table, max_q = batch
    dtype, kshape, ks, vs, dev = k.dtype, k.shape, k.stride(), v.stride(), k.get_device()
    tshape, seqs = table.shape, kv_len.shape[0] if kv_len.dim() else -1
    if not (dtype in DTYPE and v.dtype == dtype and len(kshape) == 4 and v.shape == kshape and ks[3] == 1
            and vs[3] == 1 and dev >= 0 and v.get_device() == dev and kv_len.get_device() == dev
            and table.get_device() == dev and kv_len.dtype == torch.int32 and kv_len.dim() == 1
            and kv_len.is_contiguous() and table.dtype == torch.int32 and len(tshape) == 2 and tshape[0] == seqs
            and (tshape[1] < 2 or table.stride(1) == 1)):
        _refuse(cache, batch)
    pages, heads, size, dim = kshape
    stat = kshape[:3] if weight is not None or position is not None else None
    if weight is not None and not (weight.dtype == torch.float32 and weight.shape == stat
                                   and weight.is_contiguous() and weight.get_device() == dev):
        _refuse(cache, batch)
    if position is not None and not (position.dtype == torch.int32 and position.shape == stat
                                     and position.is_contiguous() and position.get_device() == dev):
        _refuse(cache, batch)
    if offsets is not None and not (offsets.dtype == torch.int32 and offsets.dim() == 1
                                    and offsets.shape[0] == seqs + 1 and offsets.is_contiguous()
                                    and offsets.get_device() == dev):
        _refuse(cache, batch)
    width = tshape[1]
    # a table of one row may have any stride
    stride = table.stride(0)
    if seqs < 2 and stride < width:
        stride = width
    try:
        return (_CACHE.pack(k.data_ptr(), v.data_ptr(), 0 if weight is None else weight.data_ptr(),
                            0 if position is None else position.data_ptr(), ks[0], ks[1], ks[2],
                            vs[0], vs[1], vs[2], pages, size, heads, dim, DTYPE[dtype]),
                _BATCH.pack(0 if offsets is None else offsets.data_ptr(), kv_len.data_ptr(), table.data_ptr(), stride,
                            seqs, tokens, width, max_q))
    except struct.error as e:
        raise _no_fit(e, "max_q and the sizes of tensors") from None


def _no_fit(e: struct.error, what: str) -> svfsim.SvfError:
    return svfsim.SvfError(-1, f"{what} must be 32-bit integers ({e})")


def _refuse(cache: Cache, batch: Batch):
    """Says what ``_pack`` did not accept."""
    k, v, weight, position = cache
    offsets, kv_len, table, _ = batch
    _need(k.dtype in DTYPE and v.dtype == k.dtype, "k and v must both be bfloat16 or float16")
    _need(k.dim() == 4 and k.shape == v.shape, "k and v must have the shape [num_pages, kv_heads, page_size, head_dim]")
    _need(k.stride(3) == 1 and v.stride(3) == 1, "k and v must be contiguous in head_dim")
    _need(k.is_cuda, "tensors must be on a GPU")
    dev = k.get_device()
    for t, dt in ((weight, torch.float32), (position, torch.int32)):
        _need(t is None or (t.dtype == dt and t.shape == k.shape[:3] and t.is_contiguous() and t.get_device() == dev),
              "weight (float32) and position (int32) must be contiguous [num_pages, kv_heads, page_size]")
    _need(v.get_device() == dev and kv_len.get_device() == dev and table.get_device() == dev,
          "tensors must be on one GPU")
    _need(kv_len.dtype == torch.int32 and kv_len.dim() == 1 and kv_len.is_contiguous(),
          "kv_len must be contiguous int32 [seqs]")
    seqs = kv_len.shape[0]
    _need(table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == seqs
          and (table.shape[1] < 2 or table.stride(1) == 1), "page_table must be int32 [seqs, pages], rows contiguous")
    _need(False, "q_offsets must be contiguous int32 [seqs + 1] on the GPU of the cache")


def _rows(x: torch.Tensor, name: str, dtype: torch.dtype, dev: int, dim: int, heads: int = 0):
    """Strides of token and head of a [tokens, heads, head_dim] tensor of the cache's kind."""
    shape, st = x.shape, x.stride()
    if not (len(shape) == 3 and shape[2] == dim and st[2] == 1 and x.dtype == dtype and x.get_device() == dev
            and (not heads or shape[1] == heads)):
        _need(len(shape) == 3 and shape[2] == dim and st[2] == 1,
              f"{name} must be [tokens, heads, head_dim] of the cache's head_dim, contiguous in it")
        _need(False, f"{name} must have the cache's dtype, device and kv_heads")
    return st[0], st[1]


def _kind(cache: Cache):
    """What queries and outputs have to match: type, device and head size, and the key heads."""
    k = cache.k
    shape = k.shape
    if len(shape) != 4:
        _need(False, "k and v must have the shape [num_pages, kv_heads, page_size, head_dim]")
    return (k.dtype, k.get_device(), shape[3]), shape[1]


def _call(fn, dev: int, *packed, error=last_error):
    if dev == torch.cuda.current_device():
        rc = fn(*packed, _raw_stream(dev))
    else:
        with torch.cuda.device(dev):
            rc = fn(*packed, _raw_stream(dev))
    if rc != 0:
        _check(rc, error)


def _no_derivatives(*tensors: Optional[torch.Tensor]):
    """Refuses what would be lost without a word: gradients that are recorded, tangents, a place in a trace (which would hold
    this call's numbers, or its buffers without what the kernels write)."""
    level = getattr(forward_ad, "_current_level", 0) >= 0       # else no tensor has a tangent
    for t in tensors:
        if t is not None and (t.requires_grad or level):
            _need(not (t.requires_grad and torch.is_grad_enabled()),
                  "these calls have no backward pass: tensors must not require a gradient (or use torch.no_grad())")
            _need(not level or forward_ad.unpack_dual(t).tangent is None,
                  "these calls have no derivative of forward mode: tensors must not have a tangent")
    fx = sys.modules.get("torch.fx.experimental.proxy_tensor")
    if torch.jit.is_tracing() or (fx is not None and fx.get_proxy_mode() is not None):
        _need(False, "these calls cannot be traced")


def _raw_stream(dev: int) -> int:
    return torch.cuda.current_stream(dev).cuda_stream


if hasattr(torch._C, "_cuda_getCurrentRawStream"):      # the same handle without a Stream object
    _raw_stream = torch._C._cuda_getCurrentRawStream


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)     # the current one
_bound = None


class _NoBinding:
    """In the place of a binding that there is not: takes nothing, so that every call goes the long way."""

    append = attend = score = staticmethod(lambda *a: None)


def _binding():
    """The compiled binding, if it is built and of this torch."""
    global _bound
    if _bound is None:
        svfsim.load()       # torch's runtime, then the library, then what links both
        try:
            from . import _svfbinding
            why = "" if getattr(_svfbinding, "torch_version", None) == str(torch.__version__) else "it is of another torch"
        except ImportError as e:
            why = str(e)
        if why:
            warnings.warn(f"_svfbinding.so is not used ({why}): calls take some microseconds more; run __graft_entry__.build()",
                          RuntimeWarning, stacklevel=3)
        _bound = _NoBinding if why else _svfbinding
    return _bound


def _workspace(n: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    if n < 0:
        _check(int(n))
    return like.new_empty(n, dtype=torch.uint8) if n else None


def append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, rope: Optional[torch.Tensor],
           batch: Batch, cache: Cache, layout: str = "half", q_out: Optional[torch.Tensor] = None,
           axes: Optional[bytes] = None, kept: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate new queries ``q`` [tokens, heads, head_dim] and keys ``k`` [tokens,
    kv_heads, head_dim] by their ``positions`` (int32 [tokens]) and write keys and values
    ``v`` into their slots; returns the rotated queries (``q_out``, which may be
    ``q``).  ``rope`` is a table of ``rope_table`` (None: nothing is rotated);
    its width is the rotated part of a head.  Views with any strides of
    tokens and heads are taken, such as the parts of one projection's output.

    For positions with several axes ``axes`` names the axis of every pair (``pair_axes``); ``positions`` are then
    [tokens, axes], with any strides, and ``kept`` (int32 [tokens]) is what ``cache.position`` is set to in
    place of axis 0's position: the token's place in the text, which ``evict`` goes by."""
    if q.is_cuda:
        dev = _device()
        r = (_bound or _binding()).append(q, k, v, positions, rope, batch, cache, LAYOUT.get(layout), q_out, axes, kept, dev,
                                          _raw_stream(dev))
        if r is not None:
            return _check(r) if r.__class__ is int else r
    _no_derivatives(q, k, v, cache.k, cache.v, rope, q_out)
    kind, kv_heads = _kind(cache)
    dev = kind[1]
    qt, qh = _rows(q, "q", *kind)
    kt, kh = _rows(k, "k", *kind, kv_heads)
    vt, vh = _rows(v, "v", *kind, kv_heads)
    tokens, heads = q.shape[:2]
    if not (k.shape[0] == tokens and v.shape[0] == tokens):
        _need(False, "q, k and v must have as many tokens")
    if axes is not None:
        if not (positions.dtype == torch.int32 and positions.dim() == 2 and positions.shape[0] == tokens
                and positions.get_device() == dev):
            _need(False, "positions must be int32 [tokens, axes]")
        if not (kept is None or (kept.dtype == torch.int32 and kept.dim() == 1 and kept.shape[0] == tokens
                                 and kept.is_contiguous() and kept.get_device() == dev)):
            _need(False, "kept must be contiguous int32 [tokens]")
    elif not (positions.dtype == torch.int32 and positions.dim() == 1 and positions.shape[0] == tokens
              and positions.is_contiguous() and positions.get_device() == dev):
        _need(False, "positions must be contiguous int32 [tokens]")
    elif kept is not None:
        _need(False, "kept goes with axes")
    if batch.q_offsets is None or layout not in LAYOUT:
        _need(batch.q_offsets is not None, "q_offsets must not be None")
        _need(False, f"layout must be one of {tuple(LAYOUT)}")
    rows = rot = table = 0
    if rope is not None:
        if not (rope.dtype == torch.float32 and rope.dim() == 2 and rope.is_contiguous()
                and rope.get_device() == dev):
            _need(False, "rope must be contiguous float32 [positions, rot]")
        (rows, rot), table = rope.shape, rope.data_ptr()
    if q_out is None:
        q_out = torch.empty_like(q)
    elif q_out.shape != q.shape:
        _need(False, "q_out must have the shape of q")
    ot, oh = _rows(q_out, "q_out", *kind)
    a = _APPEND.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), positions.data_ptr(), table,
                     qt, qh, kt, kh, vt, vh, ot, oh, heads, rot, LAYOUT[layout], rows)
    if axes is None:
        _call(svfsim.load().svf_kv_append, dev, *_pack(cache, batch, tokens), a)
        return q_out
    if not (isinstance(axes, bytes) and len(axes) * 2 == rot and rot <= 256):
        _need(False, "axes must be bytes, one for each pair of the table (pair_axes)")
    pt, pa = positions.stride()
    x = _AXES.pack(0 if kept is None else kept.data_ptr(), pt, pa, positions.shape[1], axes)
    _call(svfsim.load().svf_kv_append_axes, dev, *_pack(cache, batch, tokens), a, x)
    return q_out


def attend(q: torch.Tensor, batch: Batch, cache: Cache, causal: bool = True, window: int = 0,
           scale: Optional[float] = None, add_weight: bool = False,
           out: Optional[torch.Tensor] = None, first: int = 0) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of the new tokens' queries ``q`` [tokens, heads, head_dim] over
    their sequences' slots: (``out`` like q, ``lse`` float32 [tokens, heads]).
    ``scale`` is 1/sqrt(head_dim) by default; ``window`` > 0 lets a token see that many
    slots up to its own, and the sequence's ``first`` slots besides; pages of slots that no token sees any more may be
    given back (-1 in the page table).  ``add_weight`` adds every slot's softmax, summed
    over the tokens and the query heads that share its key head, to
    ``cache.weight``.  A token that sees no slot has out = 0, lse = -inf."""
    if out is None and q.is_cuda:
        dev = _device()
        r = (_bound or _binding()).attend(q, batch, cache, causal, window, scale, add_weight, first, dev, _raw_stream(dev))
        if r is not None:
            return _check(r) if r.__class__ is int else r
    _no_derivatives(q, cache.k, cache.v, cache.weight if add_weight else None, out)
    kind, _ = _kind(cache)
    qt, qh = _rows(q, "q", *kind)
    if batch.q_offsets is None:
        _need(False, "q_offsets must not be None")
    tokens, heads, dim = q.shape
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape:
        _need(False, "out must have the shape of q")
    ot, oh = _rows(out, "out", *kind)
    kv, seqs = _pack(cache, batch, tokens)
    first = int(first)
    lse = q.new_empty((tokens, heads), dtype=torch.float32)
    scale = dim ** -0.5 if scale is None else float(scale)
    fixed = (qt, qh, ot, oh, scale, heads, bool(causal), int(window), bool(add_weight))
    at = (q.data_ptr(), out.data_ptr(), lse.data_ptr())
    lib = svfsim.load()
    try:
        a = _ATTEND.pack(*at, 0, 0, *fixed)
    except struct.error as e:
        raise _no_fit(e, "window and heads") from None
    if first:
        _need(0 < first < 1 << 31, "first must be >= 0, a 32-bit integer")
        need = lib.svf_kv_attend_first_workspace(kv, seqs, a, first)
    else:
        need = lib.svf_kv_attend_workspace(kv, seqs, a)
    ws = None
    if need:
        ws = _workspace(need, q)
        a = _ATTEND.pack(*at, ws.data_ptr(), need, *fixed)
    if first:
        _call(lib.svf_kv_attend_first, kind[1], kv, seqs, a, first)
    else:
        _call(lib.svf_kv_attend, kind[1], kv, seqs, a)
    return out, lse


def evict(batch: Batch, cache: Cache, budget: int, recent: int, next_position: torch.Tensor,
          first: int = 0) -> torch.Tensor:
    """Shrink every sequence that holds more than ``budget`` slots to ``budget``, each key
    head keeping the tokens of positions below ``first``, the ``recent`` newest
    before ``next_position`` (int32 [seqs]) and the rest by largest ``cache.weight``
    (ties to the lower slot).  Rows move inside the cache; returns the new lengths."""
    k, kv_len = cache.k, batch.kv_len
    _no_derivatives(k, cache.v, cache.weight)
    kv, seqs = _pack(cache, batch, 0)
    if cache.weight is None or cache.position is None:
        _need(False, "evict needs the cache's weight and position")
    if not (next_position.dtype == torch.int32 and next_position.shape == kv_len.shape
            and next_position.is_contiguous() and next_position.get_device() == k.get_device()):
        _need(False, "next_position must be contiguous int32 [seqs]")
    new_len = torch.empty_like(kv_len)
    fixed = (int(budget), int(recent), int(first))
    lib = svfsim.load()
    try:
        a = _EVICT.pack(0, 0, 0, 0, *fixed)
    except struct.error as e:
        raise _no_fit(e, "budget, recent and first") from None
    need = lib.svf_kv_evict_workspace(kv, seqs, a)
    ws = _workspace(need, k)
    a = _EVICT.pack(next_position.data_ptr(), new_len.data_ptr(), ws.data_ptr() if need else 0, need, *fixed)
    _call(lib.svf_kv_evict, k.get_device(), kv, seqs, a)
    return new_len


def pair_axes(pairs: Sequence[int], order: str = "blocks") -> bytes:
    """The axis of each pair of a head, for ``append``: axis a has ``pairs[a]`` of them, in ``blocks`` one behind the
    other or in ``turns``, a pair of each axis at a time until it has all of its pairs."""
    pairs = [int(n) for n in pairs]
    _need(1 <= len(pairs) <= MOST_AXES and min(pairs) >= 0 and sum(pairs) <= 128,
          f"pairs must be 1 .. {MOST_AXES} numbers >= 0, 128 together at most")
    _need(order in ("blocks", "turns"), "order must be 'blocks' or 'turns'")
    if order == "blocks":
        return bytes(a for a, n in enumerate(pairs) for _ in range(n))
    return bytes(a for i in range(max(pairs)) for a, n in enumerate(pairs) if i < n)


def rope_table(positions: int, rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original: int = 0, fast: float = 32.0, slow: float = 1.0, device="cuda",
               axes: Optional[bytes] = None) -> torch.Tensor:
    """Cosines and sines of ``positions`` positions for ``append``: float32 [positions,
    rot], rot/2 cosines, then rot/2 sines.  Pair i turns by position * base^(-2i/rot),
    computed in 64 bits.  For contexts ``factor`` times longer than the
    ``original`` one that a model was trained on, ``scaling`` stretches this:

    ``linear``    every frequency divided by factor (positions interpolated)
    ``base``      base times factor^(rot/(rot-2)): the slowest pair is stretched by
                  factor, the fastest not at all
    ``by-parts``  pairs that turn more than ``fast`` times within the original context stay, those
                  that turn less than ``slow`` times are divided by factor, a ramp in the
                  turns' order between them; cosines and sines times 0.1 ln(factor) + 1

    With ``axes`` (``pair_axes``) every axis has the whole range of frequencies for itself: its n pairs turn as a head
    with rot = 2n would.  Without, a pair's frequency goes by its place in the head, whichever axis it turns by.
    """
    if axes is not None:
        _need(isinstance(axes, bytes) and 2 * len(axes) == rot, "axes must be bytes, one for each pair")
        table = torch.empty((positions, rot), dtype=torch.float32, device=device)
        for a in set(axes):
            mine = [i for i, x in enumerate(axes) if x == a]
            part = rope_table(positions, 2 * len(mine), base, scaling, factor, original, fast, slow, device)
            table[:, mine + [i + len(axes) for i in mine]] = part
        return table
    _need(rot >= 2 and rot % 2 == 0 and positions >= 1, "positions must be >= 1 and rot even, >= 2")
    _need(scaling in ("none", "linear", "base", "by-parts"), f"unknown scaling {scaling!r}")
    _need(factor >= 1.0 and base > 1.0, "factor must be >= 1 and base > 1")
    i = torch.arange(rot // 2, dtype=torch.float64)
    size = 1.0
    if scaling == "base":
        _need(rot > 2, "scaling 'base' needs rot > 2")
        base = base * factor ** (rot / (rot - 2))
    freq = base ** (-2.0 * i / rot)
    if scaling == "linear":
        freq = freq / factor
    elif scaling == "by-parts":
        _need(original > 0 and fast > slow > 0, "scaling 'by-parts' needs original > 0 and fast > slow > 0")
        # the pair that turns x times within the original context
        pair = lambda x: rot * math.log(original / (x * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = math.floor(pair(fast)), math.ceil(pair(slow))     # which need not be pairs that there are
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        freq = freq * (1 - ramp) + freq / factor * ramp
        size = 0.1 * math.log(factor) + 1.0
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * freq.to(device)
    return (torch.cat((angle.cos(), angle.sin()), 1) * size).float()
