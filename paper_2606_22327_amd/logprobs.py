"""What the tokens of an answer are worth (``include/svflogprob.h``): log probabilities of given
tokens, their ranks, entropies and the best alternatives, from logits.

``score``   one row of logits and one token for each request of a step, or for each token of a prompt

Argument marshalling only, in ``csrc/svf_binding.cpp`` for ordinary arguments and here for all others: every step runs in the HIP kernels of ``libsvfsim.so``, on
torch's current stream of the tensors' device.  There are no derivatives: logits that require a gradient, where
gradients are recorded, or have a tangent of forward mode are refused, and so is a call that is being traced.  What can be checked on the host raises ``svfsim.SvfError`` (``SVF_EINVAL``).
"""

from __future__ import annotations

import struct
from typing import NamedTuple

import torch

from . import kvcache, svfsim
from .kvcache import _call, _need, _no_derivatives

DTYPE = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
TOKEN = {torch.int32: 4, torch.int64: 8}
MOST_TOP = 64

# the struct of svflogprob.h
_ARGS = struct.Struct("@8P2qf5i")


class Scores(NamedTuple):
    """``logprob``, ``entropy`` (float32) and ``rank`` (int32) [rows]; ``top_logprob`` (float32) and
    ``top_index`` (int32) [rows, top], best first."""

    logprob: torch.Tensor
    entropy: torch.Tensor
    rank: torch.Tensor
    top_logprob: torch.Tensor
    top_index: torch.Tensor


def last_error() -> str:
    return svfsim.load().svf_logprob_last_error().decode(errors="replace")


def score(logits: torch.Tensor, token: torch.Tensor, top: int = 0, scale: float = 1.0) -> Scores:
    """For each row of ``logits`` [rows, vocab] (bfloat16, float16 or float32, contiguous in vocab, rows at any
    distance) and its ``token`` (int32 or int64 [rows]): natural logarithms of softmax(scale * logits).

    ``rank`` is how many indices come before the token in the order of falling logits and, among equal ones, rising
    indices; ``top_index`` are the first ``top`` (at most 64) of that order.  ``scale`` is the inverse temperature.
    A row with a NaN or +infinity has NaN for its logarithms and its entropy, one of -infinity alone
    -infinity and 0; a token outside the vocabulary has logprob NaN and rank -1."""
    if logits.is_cuda:
        dev = kvcache._device()
        r = (kvcache._bound or kvcache._binding()).score(logits, token, top, float(scale), dev, kvcache._raw_stream(dev))
        if r is not None:
            return Scores._make(r) if r.__class__ is tuple else kvcache._check(r, last_error)
    _no_derivatives(logits)
    shape, dev = logits.shape, logits.get_device()
    if not (len(shape) == 2 and logits.dtype in DTYPE and (shape[1] < 2 or logits.stride(1) == 1) and dev >= 0):
        _need(len(shape) == 2 and logits.dtype in DTYPE, "logits must be [rows, vocab], bfloat16, float16 or float32")
        _need(logits.is_cuda, "tensors must be on a GPU")
        _need(False, "logits must be contiguous in vocab")
    rows, vocab = shape
    if not (token.dtype in TOKEN and token.dim() == 1 and token.shape[0] == rows and token.is_contiguous()
            and token.get_device() == dev):
        _need(False, "token must be contiguous int32 or int64 [rows] on the GPU of the logits")
    _need(isinstance(top, int) and 0 <= top <= min(MOST_TOP, vocab),
          f"top must be in 0 .. {MOST_TOP} and no more than vocab")
    stats = logits.new_empty((2, rows), dtype=torch.float32)
    logprob, entropy = stats.unbind()
    rank = token.new_empty(rows, dtype=torch.int32)
    top_logprob = logits.new_empty((rows, top), dtype=torch.float32)
    top_index = token.new_empty((rows, top), dtype=torch.int32)
    at = (logits.data_ptr(), token.data_ptr(), logprob.data_ptr(), entropy.data_ptr(), rank.data_ptr(),
          top_logprob.data_ptr(), top_index.data_ptr())
    fixed = (logits.stride(0), float(scale), rows, vocab, top, DTYPE[logits.dtype], TOKEN[token.dtype])
    lib = svfsim.load()
    try:
        a = _ARGS.pack(*at, 0, 0, *fixed)
    except (struct.error, OverflowError) as e:
        raise svfsim.SvfError(-1, f"sizes must be 32-bit integers and scale a 32-bit number ({e})") from None
    need = lib.svf_logprob_workspace(a)
    if need < 0:
        raise svfsim.SvfError(int(need), last_error())
    if need:
        ws = logits.new_empty(need, dtype=torch.uint8)
        a = _ARGS.pack(*at, ws.data_ptr(), need, *fixed)
    _call(lib.svf_logprob, dev, a, error=last_error)
    return Scores(logprob, entropy, rank, top_logprob, top_index)
