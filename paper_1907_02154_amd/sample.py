"""Thin Python binding over the pick of a token in libmiconv.so (``include/misample.h``): temperature, top-k, top-p and
min-p, and the draw by given random numbers.

Argument marshalling only, as in ``quant``: dtype / device / shape checks, raw device pointers, torch's current HIP
stream, and outputs and a workspace allocated here when the caller passes none.  All arithmetic runs in the library's
HIP kernels.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import miconv
from .miconv import _check, _ptr
from .quant import _CODE, _empty, _here, _matrix, _vector, _where, _workspace

_bound: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """libmiconv.so with the argument types of the sampling entry points set."""
    global _bound
    if _bound is None:
        L = miconv.lib()
        i, p, l, sz = ctypes.c_int, ctypes.c_void_p, ctypes.c_long, ctypes.c_size_t
        L.sample_tokens_workspace_bytes.argtypes = [l, l, i]
        L.sample_tokens_workspace_bytes.restype = l
        L.sample_tokens.argtypes = [l, l, i, p, l, p, p, p, p, p, p, p, p, sz, p]
        L.sample_tokens.restype = i
        _bound = L
    return _bound


def tokens_workspace_bytes(rows: int, vocab: int, dtype=torch.float32) -> int:
    """Bytes of workspace that tokens needs for logits [rows][vocab] of dtype."""
    if dtype not in _CODE:
        raise TypeError("dtype must be torch.bfloat16 or torch.float32")
    n = lib().sample_tokens_workspace_bytes(rows, vocab, _CODE[dtype])
    if n < 0:
        _check(int(n), "sample_tokens_workspace_bytes")
    return int(n)


def _operands(dev: int, rows: int, u, temperature=None, top_k=None, top_p=None, min_p=None, out=None, logprob=None, ws=None) -> None:
    """Refuses what a draw for `rows` rows on device dev cannot read, or write."""
    _vector(u, "u", dev, rows, torch.float32)
    if temperature is not None:
        _vector(temperature, "temperature", dev, rows, torch.float32)
    if top_k is not None:
        _vector(top_k, "top_k", dev, rows, torch.int32)
    if top_p is not None:
        _vector(top_p, "top_p", dev, rows, torch.float32)
    if min_p is not None:
        _vector(min_p, "min_p", dev, rows, torch.float32)
    if out is not None:
        _vector(out, "out", dev, rows, torch.int32)
    if logprob is not None:
        _vector(logprob, "logprob", dev, rows, torch.float32)


def tokens(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, out=None, logprob=None, ws=None, stream=None):
    """Draws a token of each row of logits [rows][vocab] (fp32 or bf16): (token int32 [rows], logprob fp32 [rows]), logprob
    the logarithm of the probability that the filters leave it.

    u fp32 [rows]: a random number 0 <= u < 1 for each row.  Each of temperature, top_p, min_p (fp32 [rows]) and top_k
    (int32 [rows]) may be None: temperature 1, no filter.  The first top_k tokens by logit (equal ones: the lowest index),
    of these the fewest that reach top_p of their probability, of these the ones at least min_p times as likely as the
    first; a temperature of 0 takes the first.  A row without a distribution (a NaN, an infinity, or minus infinities
    alone) gives token -1 and logprob NaN.  The exact definition: ``include/misample.h``."""
    dev = _here(logits, "logits")
    stride = _matrix(logits, "logits", dev, None, None, torch.bfloat16, torch.float32)
    rows, vocab = logits.shape
    _operands(dev, rows, u, temperature, top_k, top_p, min_p, out, logprob)
    if out is None:
        out = _empty(logits, rows, torch.int32, stream)
    if logprob is None:
        logprob = _empty(logits, rows, torch.float32, stream)
    L, code = lib(), _CODE[logits.dtype]
    wp, wn = _workspace(L.sample_tokens_workspace_bytes(rows, vocab, code), "sample_tokens", ws, logits, dev, stream)
    rc = L.sample_tokens(rows, vocab, code, logits.data_ptr(), stride, u.data_ptr(), _ptr(temperature), _ptr(top_k), _ptr(top_p),
                         _ptr(min_p), out.data_ptr(), logprob.data_ptr(), wp, wn, _where(dev, stream))
    if rc:
        _check(rc, "sample_tokens")
    return out, logprob
