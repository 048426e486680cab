"""The paged key-value cache behind the simulated budget (``include/svfkv.h``).

A schedule of ``svfsim`` counts cache slots; these calls are what one of its
steps does to a layer's cache on the GPU:

``append``   rotary positions on new queries and keys, keys and values into pages
``attend``   attention of new tokens (one or many for each sequence) over the pages
``evict``    shrinks sequences to a number of slots by accumulated attention weight
``rope_table``   cosines and sines by position, for the rotation

Argument marshalling only: every step runs in the HIP kernels of
``libsvfsim.so``, on torch's current stream of the tensors' device.  All tensors are
on one GPU.  Arguments that can be checked on the host are, and raise
``svfsim.SvfError`` (``SVF_EINVAL``); what lengths, offsets and page numbers in
device memory do is said in ``svfkv.h``.
"""

from __future__ import annotations

import math
import struct
from typing import NamedTuple, Optional, Tuple

import torch

from . import svfsim

DTYPE = {torch.bfloat16: 0, torch.float16: 1}
LAYOUT = {"half": 0, "interleaved": 1}

# the structs of svfkv.h
_CACHE = struct.Struct("@4P6q5i4x")
_BATCH = struct.Struct("@3Pq4i")
_APPEND = struct.Struct("@6P8q4i")
_ATTEND = struct.Struct("@4P5qf4i4x")
_EVICT = struct.Struct("@3Pq3i4x")


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


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _pack(cache: Cache, batch: Batch, tokens: int) -> Tuple[bytes, bytes]:
    k, v, weight, position = cache
    offsets, kv_len, table, max_q = batch
    dtype = DTYPE.get(k.dtype)
    _need(dtype is not None and v.dtype == k.dtype, "k and v must both be bfloat16 or float16")
    _need(k.dim() == 4 and k.shape == v.shape, "k and v must have the shape [num_pages, kv_heads, page_size, head_dim]")
    ks, vs = k.stride(), v.stride()
    _need(ks[3] == 1 and vs[3] == 1, "k and v must be contiguous in head_dim")
    pages, heads, size, dim = k.shape
    device = k.device
    _need(device.type == "cuda", "tensors must be on a GPU")
    for t, dt in ((weight, torch.float32), (position, torch.int32)):
        _need(t is None or (t.dtype == dt and t.shape == (pages, heads, size) and t.is_contiguous()
                            and t.device == device),
              "weight (float32) and position (int32) must be contiguous [num_pages, kv_heads, page_size]")
    _need(v.device == device and kv_len.device == device and table.device == device,
          "tensors must be on one GPU")
    _need(kv_len.dtype == torch.int32 and kv_len.dim() == 1 and kv_len.is_contiguous(),
          "kv_len must be contiguous int32 [seqs]")
    seqs = kv_len.shape[0]
    _need(table.dtype == torch.int32 and table.dim() == 2 and table.shape[0] == seqs
          and (table.shape[1] < 2 or table.stride(1) == 1), "page_table must be int32 [seqs, pages], rows contiguous")
    width = table.shape[1]
    if offsets is not None:
        _need(offsets.dtype == torch.int32 and offsets.shape == (seqs + 1,) and offsets.is_contiguous()
              and offsets.device == device, "q_offsets must be contiguous int32 [seqs + 1]")
    # a table of one row may have any stride
    stride = max(table.stride(0), width) if seqs < 2 else table.stride(0)
    return (_CACHE.pack(k.data_ptr(), v.data_ptr(), _ptr(weight), _ptr(position), ks[0], ks[1], ks[2],
                        vs[0], vs[1], vs[2], pages, size, heads, dim, dtype),
            _BATCH.pack(_ptr(offsets), kv_len.data_ptr(), table.data_ptr(), stride, seqs, tokens, width, max_q))


def _rows(x: torch.Tensor, name: str, like: torch.Tensor, tokens: int, dim: int):
    _need(x.dim() == 3 and x.shape[0] == tokens and x.shape[2] == dim and (dim < 2 or x.stride(2) == 1),
          f"{name} must be [tokens, heads, head_dim], contiguous in head_dim")
    _need(x.dtype == like.dtype and x.device == like.device, f"{name} must have the cache's dtype and device")


def _call(fn: str, device: torch.device, *packed: bytes):
    lib = svfsim.load()
    stream = torch.cuda.current_stream(device).cuda_stream
    if device.index is None or device.index == torch.cuda.current_device():
        rc = getattr(lib, fn)(*packed, stream)
    else:
        with torch.cuda.device(device):
            rc = getattr(lib, fn)(*packed, stream)
    svfsim._check(rc)


def _workspace(fn: str, device: torch.device, *packed: bytes) -> Optional[torch.Tensor]:
    n = getattr(svfsim.load(), fn)(*packed)
    if n < 0:
        svfsim._check(int(n))
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def append(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, positions: torch.Tensor, rope: Optional[torch.Tensor],
           batch: Batch, cache: Cache, layout: str = "half", q_out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Rotate new queries ``q`` [tokens, heads, head_dim] and keys ``k`` [tokens,
    kv_heads, head_dim] by their ``positions`` (int32 [tokens]) and write keys and values
    ``v`` into their slots; returns the rotated queries (``q_out``, which may be
    ``q``).  ``rope`` is a table of ``rope_table`` (None: nothing is rotated);
    its width is the rotated part of a head.  Views with any strides of
    tokens and heads are taken, such as the parts of one projection's output."""
    tokens, dim = q.shape[0] if q.dim() == 3 else -1, cache.k.shape[-1]
    for x, name in ((q, "q"), (k, "k"), (v, "v")):
        _rows(x, name, cache.k, tokens, dim)
    _need(k.shape == v.shape and k.shape[1] == cache.k.shape[1], "k and v must have the cache's kv_heads")
    _need(positions.dtype == torch.int32 and positions.shape == (tokens,) and positions.is_contiguous()
          and positions.device == q.device, "positions must be contiguous int32 [tokens]")
    _need(batch.q_offsets is not None, "q_offsets must not be None")
    _need(layout in LAYOUT, f"layout must be one of {tuple(LAYOUT)}")
    rows = rot = 0
    if rope is not None:
        _need(rope.dtype == torch.float32 and rope.dim() == 2 and rope.is_contiguous() and rope.device == q.device,
              "rope must be contiguous float32 [positions, rot]")
        rows, rot = rope.shape
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _rows(q_out, "q_out", cache.k, tokens, dim)
        _need(q_out.shape == q.shape, "q_out must have the shape of q")
    a = _APPEND.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), positions.data_ptr(), _ptr(rope),
                     q.stride(0), q.stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1),
                     q_out.stride(0), q_out.stride(1), q.shape[1], rot, LAYOUT[layout], rows)
    _call("svf_kv_append", q.device, *_pack(cache, batch, tokens), a)
    return q_out


def attend(q: torch.Tensor, batch: Batch, cache: Cache, causal: bool = True, window: int = 0,
           scale: Optional[float] = None, add_weight: bool = False,
           out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of the new tokens' queries ``q`` [tokens, heads, head_dim] over
    their sequences' slots: (``out`` like q, ``lse`` float32 [tokens, heads]).
    ``scale`` is 1/sqrt(head_dim) by default; ``window`` > 0 lets a token see that many
    slots up to its own.  ``add_weight`` adds every slot's softmax, summed
    over the tokens and the query heads that share its key head, to
    ``cache.weight``.  A token that sees no slot has out = 0, lse = -inf."""
    tokens, dim = q.shape[0] if q.dim() == 3 else -1, cache.k.shape[-1]
    _rows(q, "q", cache.k, tokens, dim)
    _need(batch.q_offsets is not None, "q_offsets must not be None")
    heads = q.shape[1]
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    else:
        _rows(out, "out", cache.k, tokens, dim)
        _need(out.shape == q.shape, "out must have the shape of q")
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device)
    packed = _pack(cache, batch, tokens)
    scale = 1.0 / math.sqrt(dim) if scale is None else float(scale)

    def args(ws):
        return _ATTEND.pack(q.data_ptr(), out.data_ptr(), lse.data_ptr(), _ptr(ws), 0 if ws is None else ws.numel(),
                            q.stride(0), q.stride(1), out.stride(0), out.stride(1), scale, heads, bool(causal),
                            int(window), bool(add_weight))

    a = args(None)
    ws = _workspace("svf_kv_attend_workspace", q.device, *packed, a)
    _call("svf_kv_attend", q.device, *packed, a if ws is None else args(ws))
    return out, lse


def evict(batch: Batch, cache: Cache, budget: int, recent: int, next_position: torch.Tensor,
          first: int = 0) -> torch.Tensor:
    """Shrink every sequence that holds more than ``budget`` slots to ``budget``, each key
    head keeping the tokens of positions below ``first``, the ``recent`` newest
    before ``next_position`` (int32 [seqs]) and the rest by largest ``cache.weight``
    (ties to the lower slot).  Rows move inside the cache; returns the new lengths."""
    k, kv_len = cache.k, batch.kv_len
    packed = _pack(cache, batch, 0)
    _need(cache.weight is not None and cache.position is not None, "evict needs the cache's weight and position")
    _need(next_position.dtype == torch.int32 and next_position.shape == kv_len.shape
          and next_position.is_contiguous() and next_position.device == k.device,
          "next_position must be contiguous int32 [seqs]")
    new_len = torch.empty_like(kv_len)

    def args(ws):
        return _EVICT.pack(next_position.data_ptr(), new_len.data_ptr(), _ptr(ws), 0 if ws is None else ws.numel(),
                           int(budget), int(recent), int(first))

    ws = _workspace("svf_kv_evict_workspace", k.device, *packed, args(None))
    _call("svf_kv_evict", k.device, *packed, args(ws))
    return new_len


def rope_table(positions: int, rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
               original: int = 0, fast: float = 32.0, slow: float = 1.0, device="cuda") -> torch.Tensor:
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
    """
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
        lo, hi = math.floor(pair(fast)), math.ceil(pair(slow))
        lo, hi = max(lo, 0), min(hi, rot // 2 - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        freq = freq * (1 - ramp) + freq / factor * ramp
        size = 0.1 * math.log(factor) + 1.0
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * freq.to(device)
    return (torch.cat((angle.cos(), angle.sin()), 1) * size).float()
