"""Torch-facing operators of the language model around the mixer: linear
attention with a decay per head, the scaled embedding lookup and counter-based
dropout.

Marshalling only: each call runs the library's kernels (``include/bcmt.h``) on
the current CUDA stream.  ``linear_attention``, ``embedding`` and ``dropout``
are differentiable (the last two, which are linear, any number of times; a second
derivative of linear attention raises); the ``*_forward`` / ``*_backward`` / ``*_step`` functions
are the bare calls.  Arguments that the library would misread (devices, types,
shapes, layouts) raise ``ValueError``; what the library refuses raises
``bcmt.BCMTError``.
"""

from __future__ import annotations

import ctypes
import functools
import math
from typing import Optional, Tuple

import torch
from torch.autograd.function import once_differentiable
from torch.autograd.graph import increment_version

from . import bcmt as C

_DTYPES = {torch.bfloat16: C.BCMT_BF16, torch.float32: C.BCMT_F32}
_F32 = torch.float32

# The calls below take a few microseconds of kernel time at small sizes, so
# their own host time counts: checks format their message only when they fail,
# parameters are built once per shape, and the stream is read as a raw handle.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) \
    or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _device(t: torch.Tensor) -> torch.device:
    dev = t.device
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on a CUDA device, not {dev}")
    return dev


def _dtype(t: torch.Tensor, name: str) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise ValueError(f"{name} must be bfloat16 or float32, not {t.dtype}")
    return dt


def _check(t, name, shape, dtype, dev):
    if t.shape != shape or t.dtype != dtype or t.device != dev:
        raise ValueError(f"{name} must be {dtype} {tuple(shape)} on {dev}, not {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")


def _on_its_device(fn):
    """Runs fn with its first tensor's device current (a switch only where it is not)."""
    @functools.wraps(fn)
    def call(*args, **kwargs):
        first = args[0] if args else next(
            (t for t in kwargs.values() if isinstance(t, torch.Tensor)), None)
        if not isinstance(first, torch.Tensor):
            raise ValueError(f"a tensor is needed, not {type(first).__name__}")
        if first.is_cuda and first.get_device() != _current_device():
            with torch.cuda.device(first.device):
                return fn(*args, **kwargs)
        return fn(*args, **kwargs)
    return call


def _dense(t):
    """t dense and 16-byte aligned (copied where it is not); None stays None."""
    if t is None:
        return None
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _number(x, name: str) -> Optional[float]:
    """x as a Python float (None stays None): the plans are kept by value, and what a
    call reads from a tensor or array must not change with it later."""
    if type(x) is float or x is None:
        return x
    if isinstance(x, torch.Tensor) and x.requires_grad:
        raise ValueError(f"{name} is a constant here: it gets no gradient")
    return float(x)


def _buffer(nbytes: int, device) -> torch.Tensor:
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


# ------------------------------------------------------------ linear attention
def _is_rows(stride, shape) -> bool:
    B, T, H, dh = shape
    sb, st, sh, sd = stride
    ld = st if T > 1 else sb if B > 1 else H * dh
    return (sd == 1 and (H == 1 or sh == dh) and (B == 1 or sb == T * ld) and ld >= H * dh
            and ld % 8 == 0)


def _rows(t: torch.Tensor, shape) -> Tuple[torch.Tensor, int, int]:
    """t [B, T, H, dh] as rows of one stride: (tensor, address, stride in elements).
    A slice of a projection's output is taken as it is, anything else copied."""
    stride = t.stride()
    ptr = t.data_ptr()
    if ptr % 16 or not _is_rows(stride, shape):
        t = _dense(t)
        return t, t.data_ptr(), shape[2] * shape[3]
    return t, ptr, stride[1] if shape[1] > 1 else stride[0] if shape[0] > 1 else shape[2] * shape[3]


@functools.lru_cache(maxsize=4096)
def _linattn_plan(B, T, H, dh, dt, scale, backward):
    """(parameters by reference, bytes of workspace; 0 where the call needs none)."""
    p = C.bcmt_linattn_params(B, T, H, dh, dt, 0, 1.0 / math.sqrt(dh) if scale is None else scale)
    n = C.bcmt_linattn_workspace_size(p, backward)
    return ctypes.byref(p), n if n > 256 else 0


def _linattn_check(q, k, v, decay, lengths, state):
    dev = _device(q)
    shape, dtype = q.shape, q.dtype
    if len(shape) != 4:
        raise ValueError(f"q must be [B, T, H, dh], not {tuple(shape)}")
    dt = _dtype(q, "q")
    if k.shape != shape or k.dtype != dtype or k.device != dev:
        _check(k, "k", shape, dtype, dev)
    if v.shape != shape or v.dtype != dtype or v.device != dev:
        _check(v, "v", shape, dtype, dev)
    B, T, H, dh = shape
    _check(decay, "decay", (H,), _F32, dev)
    if decay.requires_grad:
        raise ValueError("decay is a constant here: it gets no gradient")
    if lengths is not None:
        _check(lengths, "lengths", (B,), torch.int32, dev)
        lengths = lengths.contiguous()
    if state is not None:
        _check(state, "state", (B, H, dh, dh), _F32, dev)
        state = _dense(state)
    return dev, dt, decay.contiguous(), lengths, state


def _address(t):
    return None if t is None else t.data_ptr()


@_on_its_device
def linear_attention_forward(q, k, v, decay, scale: Optional[float] = None, lengths=None,
                             state=None, state_out=None):
    """(o, state_out) of ``S_t = a S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t``.

    q, k, v [B, T, H, dh] (bf16 or fp32; slices of one projection's rows are read
    in place), decay [H] fp32, each in [0, 1] (others are reported by
    ``bcmt.bcmt_device_status``), lengths [B] int32 (tokens per sequence, default
    T), state [B, H, dh, dh] fp32 (default zero).  scale defaults to
    1/sqrt(dh).  state_out: where the last state goes (default a new tensor; may
    be ``state``); autograd sees it as modified in place.  Tokens past a sequence's
    length give zero rows."""
    dev, dt, decay, lengths, state = _linattn_check(q, k, v, decay, lengths, state)
    shape = q.shape
    B, T, H, dh = shape
    given = state_out
    if state_out is None:
        state_out = torch.empty((B, H, dh, dh), dtype=_F32, device=dev)
    elif state_out is not state:
        _check(state_out, "state_out", (B, H, dh, dh), _F32, dev)
        if not state_out.is_contiguous():
            raise ValueError("state_out must be dense")
    p, nbytes = _linattn_plan(B, T, H, dh, dt, _number(scale, "scale"), False)
    (q, pq, lq), (k, pk, lk), (v, pv, lv) = _rows(q, shape), _rows(k, shape), _rows(v, shape)
    o = torch.empty(shape, dtype=q.dtype, device=dev)
    ws = _buffer(nbytes, dev) if nbytes else None
    C.check(C.LIB.bcmt_linattn_forward(
        p, pq, lq, pk, lk, pv, lv, decay.data_ptr(), _address(lengths), _address(state),
        o.data_ptr(), H * dh, state_out.data_ptr(), _address(ws), _raw_stream(dev.index)))
    if given is not None:   # written through its address, which autograd cannot see
        increment_version(given)
    return o, state_out


@_on_its_device
def linear_attention_backward(do, q, k, v, decay, scale: Optional[float] = None, lengths=None,
                              state=None, dstate=None, need_dstate: Optional[bool] = None):
    """(dq, dk, dv, d_state) from the forward's inputs, do [B, T, H, dh] and the
    gradient dstate of the last state (default zero).  d_state, the gradient of
    the first state, is computed when a state was given (or by need_dstate),
    else None."""
    dev, dt, decay, lengths, state = _linattn_check(q, k, v, decay, lengths, state)
    shape = q.shape
    _check(do, "do", shape, q.dtype, dev)
    B, T, H, dh = shape
    D = H * dh
    if need_dstate is None:
        need_dstate = state is not None
    if dstate is not None:
        _check(dstate, "dstate", (B, H, dh, dh), _F32, dev)
        dstate = _dense(dstate)
    p, nbytes = _linattn_plan(B, T, H, dh, dt, _number(scale, "scale"), True)
    (do, pd, ldo), (q, pq, lq) = _rows(do, shape), _rows(q, shape)
    (k, pk, lk), (v, pv, lv) = _rows(k, shape), _rows(v, shape)
    dq, dk, dv = (torch.empty(shape, dtype=q.dtype, device=dev) for _ in range(3))
    ds = torch.empty((B, H, dh, dh), dtype=_F32, device=dev) if need_dstate else None
    ws = _buffer(nbytes, dev) if nbytes else None
    C.check(C.LIB.bcmt_linattn_backward(
        p, pd, ldo, pq, lq, pk, lk, pv, lv, decay.data_ptr(), _address(lengths), _address(state),
        _address(dstate), dq.data_ptr(), D, dk.data_ptr(), D, dv.data_ptr(), D, _address(ds),
        _address(ws), _raw_stream(dev.index)))
    return dq, dk, dv, ds


def linear_attention_step(q, k, v, decay, state, scale: Optional[float] = None, active=None,
                          state_out=None):
    """One token of each sequence: q, k, v [B, 1, H, dh]; updates ``state`` (in
    place unless state_out is given) and returns o [B, 1, H, dh].  active [B]
    int32: sequences with 0 keep their state and get a zero row.  A state that a
    differentiable call read cannot be updated in place before that call's
    backward (which then raises): pass a copy or a state_out."""
    if q.dim() != 4 or q.shape[1] != 1 or state is None:
        raise ValueError(f"q must be [B, 1, H, dh], not {tuple(q.shape)}, and state a tensor")
    return linear_attention_forward(q, k, v, decay, scale, active, state,
                                    state if state_out is None else state_out)[0]


class LinearAttention(torch.autograd.Function):
    """(o, last state) with q, k, v and the first state as differentiable inputs."""

    @staticmethod
    def forward(ctx, q, k, v, decay, scale, lengths, state):
        o, last = linear_attention_forward(q, k, v, decay, scale, lengths, state)
        ctx.save_for_backward(q, k, v, decay, lengths, state)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        return o, last

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dlast):
        q, k, v, decay, lengths, state = ctx.saved_tensors
        if do is None and dlast is None:
            return (None,) * 7
        if do is None:
            do = torch.zeros_like(q, memory_format=torch.contiguous_format)
        dq, dk, dv, ds = linear_attention_backward(
            do, q, k, v, decay, ctx.scale, lengths, state, dlast,
            need_dstate=state is not None and ctx.needs_input_grad[6])
        return dq, dk, dv, None, None, None, ds


def linear_attention(q, k, v, decay, scale: Optional[float] = None, lengths=None, state=None):
    """Differentiable ``linear_attention_forward``: (o, last state)."""
    return LinearAttention.apply(q, k, v, decay, _number(scale, "scale"), lengths, state)


# ------------------------------------------------------------------- embedding
@functools.lru_cache(maxsize=4096)
def _embedding_plan(N, V, D, dt, id_bytes, scale):
    p = C.bcmt_embedding_params(N, V, D, dt, id_bytes, 0, scale)
    return ctypes.byref(p), max(256, C.bcmt_embedding_workspace_size(p))


def _ids(ids, dev):
    if ids.dtype != torch.int64 and ids.dtype != torch.int32:
        raise ValueError(f"ids must be int32 or int64, not {ids.dtype}")
    if ids.device != dev:
        raise ValueError(f"ids must be on {dev}, not {ids.device}")
    return ids.contiguous()


@_on_its_device
def embedding_forward(ids, weight, scale: float = 1.0):
    """``scale * weight[ids]``: ids of any shape (int32 or int64), weight [V, D].
    Ids outside the table give zero rows and are reported by
    ``bcmt.bcmt_device_status``."""
    dev = _device(weight)
    if weight.dim() != 2:
        raise ValueError(f"weight must be [V, D], not {tuple(weight.shape)}")
    ids = _ids(ids, dev)
    V, D = weight.shape
    p, _ = _embedding_plan(ids.numel(), V, D, _dtype(weight, "weight"), ids.element_size(),
                           _number(scale, "scale"))
    out = torch.empty((*ids.shape, D), dtype=weight.dtype, device=dev)
    weight = _dense(weight)
    C.check(C.LIB.bcmt_embedding_forward(p, ids.data_ptr(), weight.data_ptr(), out.data_ptr(),
                                         _raw_stream(dev.index)))
    return out


@_on_its_device
def embedding_backward(ids, dout, V: int, scale: float = 1.0):
    """Gradient [V, D] of the table from dout [*ids.shape, D]."""
    dev = _device(dout)
    if dout.shape[:-1] != ids.shape:
        raise ValueError(f"dout must be [*ids.shape, D], not {tuple(dout.shape)}")
    ids = _ids(ids, dev)
    D = dout.shape[-1]
    p, nbytes = _embedding_plan(ids.numel(), V, D, _dtype(dout, "dout"), ids.element_size(),
                                _number(scale, "scale"))
    dw = torch.empty((V, D), dtype=dout.dtype, device=dev)
    ws = _buffer(nbytes, dev)
    dout = _dense(dout)
    C.check(C.LIB.bcmt_embedding_backward(p, ids.data_ptr(), dout.data_ptr(), dw.data_ptr(),
                                          ws.data_ptr(), _raw_stream(dev.index)))
    return dw


class Embedding(torch.autograd.Function):
    """``scale * weight[ids]`` with the table as the differentiable input."""

    @staticmethod
    def forward(ctx, ids, weight, scale):
        ctx.save_for_backward(ids)
        ctx.V, ctx.scale = weight.shape[0], scale
        return embedding_forward(ids, weight, scale)

    @staticmethod
    def backward(ctx, dout):
        ids, = ctx.saved_tensors
        # with a graph of its own where one is wanted (create_graph)
        grad = EmbeddingGrad.apply if torch.is_grad_enabled() else embedding_backward
        return None, grad(ids, dout, ctx.V, ctx.scale), None


class EmbeddingGrad(torch.autograd.Function):
    """The table's gradient as a function of dout; its own gradient is the lookup."""

    @staticmethod
    def forward(ctx, ids, dout, V, scale):
        ctx.save_for_backward(ids)
        ctx.scale = scale
        return embedding_backward(ids, dout, V, scale)

    @staticmethod
    def backward(ctx, ddw):
        ids, = ctx.saved_tensors
        return None, embedding(ids, ddw, ctx.scale), None, None


def embedding(ids, weight, scale: float = 1.0):
    """Differentiable ``embedding_forward``."""
    return Embedding.apply(ids, weight, _number(scale, "scale"))


# --------------------------------------------------------------------- dropout
@_on_its_device
def _dropout_call(x, p, seed, offset, residual, step):
    dev = _device(x)
    dt = _dtype(x, "x")
    if residual is not None:
        _check(residual, "residual", x.shape, x.dtype, dev)
        residual = _dense(residual)
    if step is not None:
        if step.dtype != torch.int64 or step.numel() != 1 or step.device != dev:
            raise ValueError(f"step must be one int64 on {dev}")
        step = step.data_ptr()
    x = _dense(x)
    y = torch.empty(x.shape, dtype=x.dtype, device=dev)
    mask = (1 << 64) - 1
    prm = C.bcmt_dropout_params(x.numel(), dt, 0, _number(p, "p"), int(seed) & mask,
                                 int(offset) & mask, step)
    C.check(C.LIB.bcmt_dropout(ctypes.byref(prm), x.data_ptr(), _address(residual), y.data_ptr(),
                               _raw_stream(dev.index)))
    return y


def dropout_forward(x, p: float, seed: int, offset: int, residual=None, step=None):
    """``[residual +] keep * x / (1 - p)``, the mask a function of (seed, offset +
    step) and the element's index, its rate 1 - p to 2^-17 (where that is too coarse
    for 1 / (1 - p), near p = 1, the scale is the mask's own); step: an int64 on the device (for captured
    graphs), default 0."""
    return _dropout_call(x, p, seed, offset, residual, step)


def dropout_backward(dy, p: float, seed: int, offset: int, step=None):
    """Gradient of x: the same mask on dy (that of residual is dy itself)."""
    return _dropout_call(dy, p, seed, offset, None, step)


class Dropout(torch.autograd.Function):
    """``[residual +] dropout(x)``; the backward recomputes the mask."""

    @staticmethod
    def forward(ctx, x, p, seed, offset, residual, step):
        ctx.args = (p, seed, offset)
        # the counter may move on before the backward: keep its value of now
        ctx.step = None if step is None else step.clone()
        return dropout_forward(x, p, seed, offset, residual, step)

    @staticmethod
    def backward(ctx, dy):
        dx = None
        if ctx.needs_input_grad[0]:
            # with a graph of its own where one is wanted (create_graph): the same mask
            dx = dropout(dy, *ctx.args, step=ctx.step) if torch.is_grad_enabled() \
                else dropout_backward(dy, *ctx.args, step=ctx.step)
        return dx, None, None, None, dy if ctx.needs_input_grad[4] else None, None


def dropout(x, p: float, seed: int, offset: int, residual=None, step=None):
    """Differentiable ``dropout_forward``."""
    return Dropout.apply(x, _number(p, "p"), int(seed), int(offset), residual, step)
