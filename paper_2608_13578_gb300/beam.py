"""A step of beam search: the selection over beams and vocabulary, and the
reordering of the beams' states.

Marshalling only, as in ``lm_ops``; nothing here is differentiable.  Arguments that
the library would misread raise ``ValueError``; what the library refuses raises
``bcmt.BCMTError``.
"""

from __future__ import annotations

import ctypes
import functools
from array import array
from typing import Optional

import torch
from torch.autograd.graph import increment_version

from . import bcmt as C
from .lm_ops import _address, _buffer, _check, _current_device, _device, _dtype, _on_its_device, \
    _raw_stream


@functools.lru_cache(maxsize=4096)
def _plan(N, K, V, dt, eos, ld):
    p = C.bcmt_beam_params(N, K, V, dt, eos, 0, ld)
    return ctypes.byref(p), C.bcmt_beam_workspace_size(p)


@_on_its_device
def beam_select(logits, scores, finished=None, eos: Optional[int] = None):
    """(scores, parents, tokens, finished) of the K best continuations of each search, the
    best first: candidates ``scores[n, k] + log_softmax(logits[n, k])[v]``, equal ones in the
    order of k V + v.  Candidates of different beams that are nearer than (6 ln V + 50) 2^-24
    may change places: most of each row's sum of exponentials is taken in fp32.

    logits [N, K, V] (bf16 or fp32, 1 <= K <= 32; rows of one stride, as in a slice of the last
    tokens, are read in place; -inf: ruled out), scores [N, K] fp32 (-inf: no beam there, as
    all but the first of a new search), finished [N, K] bool: beams that have ended, which
    keep their score and get the token ``eos``.  Returns [N, K] fp32, int64, int64 and bool.
    A NaN or +inf takes its beam out and is reported by ``bcmt.bcmt_device_status``."""
    dev = _device(logits)
    if logits.dim() != 3:
        raise ValueError(f"logits must be [N, K, V], not {tuple(logits.shape)}")
    if (logits.requires_grad or scores.requires_grad) and torch.is_grad_enabled():
        raise ValueError("beam_select is not differentiable: call it under torch.no_grad")
    dt = _dtype(logits, "logits")
    N, K, V = logits.shape
    _check(scores, "scores", (N, K), torch.float32, dev)
    if finished is not None:
        _check(finished, "finished", (N, K), torch.bool, dev)
        if eos is None:
            raise ValueError("finished beams need an end token eos")
        finished = finished.contiguous()
    if eos is not None and not 0 <= int(eos) < V:
        raise ValueError(f"eos = {eos} must be in 0 .. {V - 1}")
    sn, sk, sv = logits.stride()
    ld = sk if K > 1 else sn if N > 1 else V
    if (V > 1 and sv != 1) or ld < V or (N > 1 and K > 1 and sn != K * sk):
        logits, ld = logits.contiguous(), V
    p, nbytes = _plan(N, K, V, dt, -1 if eos is None else int(eos), ld)
    scores = scores.contiguous()
    out = torch.empty((N, K), dtype=torch.float32, device=dev)
    parents, tokens = (torch.empty((N, K), dtype=torch.int64, device=dev) for _ in range(2))
    ended = torch.empty((N, K), dtype=torch.bool, device=dev)
    ws = _buffer(max(256, nbytes), dev)
    C.check(C.LIB.bcmt_beam_select(
        p, logits.data_ptr(), scores.data_ptr(), _address(finished), out.data_ptr(),
        parents.data_ptr(), tokens.data_ptr(), ended.data_ptr(), ws.data_ptr(),
        _raw_stream(dev.index)))
    return out, parents, tokens, ended


def beam_reorder(tensors, parents, out=None):
    """``t[n, parents[n, k]]`` for every t of ``tensors`` ([N, K, ...] or [N * K, ...], any type):
    a list of new tensors, or those of ``out`` (dense; they may not share memory with ``tensors``,
    ``parents`` or each other).  A parent outside its beams gives zeros and is reported by
    ``bcmt.bcmt_device_status``."""
    if not isinstance(parents, torch.Tensor):
        raise ValueError(f"parents must be a tensor, not {type(parents).__name__}")
    dev = _device(parents)
    if dev.index != _current_device():
        with torch.cuda.device(dev):
            return beam_reorder(tensors, parents, out)
    if parents.dim() != 2 or parents.dtype != torch.int64:
        raise ValueError(f"parents must be int64 [N, K], not {parents.dtype} {tuple(parents.shape)}")
    N, K = parents.shape
    NK, at, index = N * K, dev.index, parents.get_device()
    parents = parents.contiguous()
    grad, rows, table = torch.is_grad_enabled(), [], array("q")
    tensors = list(tensors)
    fresh = out is None
    out = [None] * len(tensors) if fresh else list(out)
    if len(out) != len(tensors):
        raise ValueError(f"out must have {len(tensors)} tensors, not {len(out)}")
    for i, t in enumerate(tensors):
        shape = t.shape
        n = t.numel()
        if (t.get_device() != index or not shape
                or not (shape[0] == NK or (shape[0] == N and len(shape) > 1 and shape[1] == K))):
            raise ValueError(f"tensors must be [N, K, ...] or [N K, ...] on {dev}, not "
                             f"{tuple(shape)} on {t.device}")
        if grad and t.requires_grad:
            raise ValueError("beam_reorder is not differentiable: call it under torch.no_grad")
        if not t.is_contiguous():
            t = t.contiguous()
            rows.append(t)   # alive until the launch
        if fresh:
            o = out[i] = torch.empty_like(t)
        else:
            o = out[i]
            if (o.shape != shape or o.dtype is not t.dtype or o.get_device() != index
                    or not o.is_contiguous()):
                _check(o, "out", shape, t.dtype, dev)
                raise ValueError("out must be dense")
        table.extend((t.data_ptr(), o.data_ptr(), n // NK * t.element_size() if n else 0))
    if not out or NK == 0:
        return out
    C.check(C.LIB.bcmt_beam_reorder(parents.data_ptr(), N, K, table.buffer_info()[0], len(out), 0,
                                    _raw_stream(at)))
    if not fresh:
        increment_version(out)   # written through its address, which autograd cannot see
    return out
