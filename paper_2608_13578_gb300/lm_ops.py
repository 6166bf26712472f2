"""Torch-facing operators of the language model around the mixer: linear
attention with a decay per head, the scaled embedding lookup and counter-based
dropout.

Marshalling only: each call runs the library's kernels (``include/bcmt.h``) on
the current CUDA stream.  ``linear_attention``, ``embedding`` and ``dropout``
are differentiable; the ``*_forward`` / ``*_backward`` / ``*_step`` functions
are the bare calls.  Arguments that the library would misread (devices, types,
shapes, layouts) raise ``ValueError``; what the library refuses raises
``bcmt.BCMTError``.
"""

from __future__ import annotations

import math
from typing import Optional, Tuple

import torch

from . import bcmt as C

_DTYPES = {torch.bfloat16: C.BCMT_BF16, torch.float32: C.BCMT_F32}


def _need(ok: bool, msg: str):
    if not ok:
        raise ValueError(msg)


def _dtype(t: torch.Tensor, name: str) -> int:
    _need(t.dtype in _DTYPES, f"{name} must be bfloat16 or float32, not {t.dtype}")
    return _DTYPES[t.dtype]


def _on(device, **tensors):
    _need(device.type == "cuda", f"tensors must be on a CUDA device, not {device}")
    for name, t in tensors.items():
        _need(t is None or t.device == device, f"{name} must be on {device}")


def _dense(t):
    """t dense and 16-byte aligned (copied where it is not); None stays None."""
    if t is None:
        return None
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _buffer(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(256, nbytes), dtype=torch.uint8, device=device)


# ------------------------------------------------------------ linear attention
def _rows(t: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """t [B, T, H, dh] as rows of one stride (a slice of a projection's output as
    it is, anything else copied), and that stride in elements."""
    B, T, H, dh = t.shape
    ld = t.stride(1) if T > 1 else (t.stride(0) if B > 1 else H * dh)
    ok = (t.stride(3) == 1 and (H == 1 or t.stride(2) == dh) and (B == 1 or t.stride(0) == T * ld)
          and ld >= H * dh and ld % 8 == 0 and t.data_ptr() % 16 == 0)
    return (t, ld) if ok else (_dense(t), H * dh)


def _linattn_check(q, k, v, decay, lengths, state, T=None):
    _need(q.dim() == 4, f"q must be [B, T, H, dh], not {tuple(q.shape)}")
    B, T, H, dh = q.shape
    _on(q.device, k=k, v=v, decay=decay, lengths=lengths, state=state)
    dt = _dtype(q, "q")
    for name, t in (("k", k), ("v", v)):
        _need(t.shape == q.shape and t.dtype == q.dtype,
              f"{name} must have q's shape and type: {tuple(t.shape)} {t.dtype}")
    _need(decay.shape == (H,) and decay.dtype == torch.float32,
          f"decay must be float32 [{H}], not {decay.dtype} {tuple(decay.shape)}")
    _need(not decay.requires_grad, "decay is a constant here: it gets no gradient")
    if lengths is not None:
        _need(lengths.shape == (B,) and lengths.dtype == torch.int32,
              f"lengths must be int32 [{B}], not {lengths.dtype} {tuple(lengths.shape)}")
    if state is not None:
        _need(state.shape == (B, H, dh, dh) and state.dtype == torch.float32,
              f"state must be float32 {(B, H, dh, dh)}, not {state.dtype} {tuple(state.shape)}")
    return dt


def _linattn_params(q, scale, dt):
    B, T, H, dh = q.shape
    return C.bcmt_linattn_params(B, T, H, dh, dt, 0, 1.0 / math.sqrt(dh) if scale is None else scale)


def linear_attention_forward(q, k, v, decay, scale: Optional[float] = None, lengths=None,
                             state=None, state_out=None):
    """(o, state_out) of ``S_t = a S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t``.

    q, k, v [B, T, H, dh] (bf16 or fp32; slices of one projection's rows are read
    in place), decay [H] fp32, lengths [B] int32 (tokens per sequence, default
    T), state [B, H, dh, dh] fp32 (default zero).  scale defaults to
    1/sqrt(dh).  state_out: where the last state goes (default a new tensor; may
    be ``state``).  Tokens past a sequence's length give zero rows."""
    dt = _linattn_check(q, k, v, decay, lengths, state)
    if state_out is not None:
        B, T, H, dh = q.shape
        _need(state_out.shape == (B, H, dh, dh) and state_out.dtype == torch.float32
              and state_out.is_contiguous() and state_out.device == q.device,
              f"state_out must be dense float32 {(B, H, dh, dh)} on {q.device}")
    with torch.cuda.device(q.device):
        p = _linattn_params(q, scale, dt)
        (q, lq), (k, lk), (v, lv) = _rows(q), _rows(k), _rows(v)
        B, T, H, dh = q.shape
        o = torch.empty(B, T, H, dh, dtype=q.dtype, device=q.device)
        if state_out is None:
            state_out = torch.empty(B, H, dh, dh, dtype=torch.float32, device=q.device)
        ws = _buffer(C.bcmt_linattn_workspace_size(p, False), q.device)
        C.bcmt_linattn_forward(p, q, lq, k, lk, v, lv, _dense(decay), _dense(lengths),
                               _dense(state), o, H * dh, state_out, ws)
    return o, state_out


def linear_attention_backward(do, q, k, v, decay, scale: Optional[float] = None, lengths=None,
                              state=None, dstate=None, need_dstate: Optional[bool] = None):
    """(dq, dk, dv, d_state) from the forward's inputs, do [B, T, H, dh] and the
    gradient dstate of the last state (default zero).  d_state, the gradient of
    the first state, is computed when a state was given (or by need_dstate),
    else None."""
    dt = _linattn_check(q, k, v, decay, lengths, state)
    _need(do.shape == q.shape and do.dtype == q.dtype and do.device == q.device,
          f"do must have q's shape, type and device: {tuple(do.shape)} {do.dtype}")
    if dstate is not None:
        B, T, H, dh = q.shape
        _need(dstate.shape == (B, H, dh, dh) and dstate.dtype == torch.float32
              and dstate.device == q.device, f"dstate must be float32 {(B, H, dh, dh)}")
    if need_dstate is None:
        need_dstate = state is not None
    with torch.cuda.device(q.device):
        p = _linattn_params(q, scale, dt)
        (do, ldo), (q, lq), (k, lk), (v, lv) = _rows(do), _rows(q), _rows(k), _rows(v)
        B, T, H, dh = q.shape
        dq, dk, dv = (torch.empty(B, T, H, dh, dtype=q.dtype, device=q.device) for _ in range(3))
        ds = torch.empty(B, H, dh, dh, dtype=torch.float32, device=q.device) if need_dstate else None
        ws = _buffer(C.bcmt_linattn_workspace_size(p, True), q.device)
        C.bcmt_linattn_backward(p, do, ldo, q, lq, k, lk, v, lv, _dense(decay), _dense(lengths),
                                _dense(state), _dense(dstate), dq, H * dh, dk, H * dh, dv, H * dh,
                                ds, ws)
    return dq, dk, dv, ds


def linear_attention_step(q, k, v, decay, state, scale: Optional[float] = None, active=None,
                          state_out=None):
    """One token of each sequence: q, k, v [B, 1, H, dh]; updates ``state`` (in
    place unless state_out is given) and returns o [B, 1, H, dh].  active [B]
    int32: sequences with 0 keep their state and get a zero row."""
    _need(q.dim() == 4 and q.shape[1] == 1, f"q must be [B, 1, H, dh], not {tuple(q.shape)}")
    if state_out is None:
        state_out = state
    return linear_attention_forward(q, k, v, decay, scale, active, state, state_out)[0]


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
    return LinearAttention.apply(q, k, v, decay, scale, lengths, state)


# ------------------------------------------------------------------- embedding
def _embedding_params(ids, V, D, dt, scale):
    _need(ids.dtype in (torch.int32, torch.int64), f"ids must be int32 or int64, not {ids.dtype}")
    return C.bcmt_embedding_params(ids.numel(), V, D, dt, ids.element_size(), 0, scale)


def embedding_forward(ids, weight, scale: float = 1.0):
    """``scale * weight[ids]``: ids of any shape (int32 or int64), weight [V, D].
    Ids outside the table give zero rows and are reported by
    ``bcmt.bcmt_device_status``."""
    _need(weight.dim() == 2, f"weight must be [V, D], not {tuple(weight.shape)}")
    _on(weight.device, ids=ids)
    V, D = weight.shape
    with torch.cuda.device(weight.device):
        p = _embedding_params(ids, V, D, _dtype(weight, "weight"), scale)
        out = torch.empty(*ids.shape, D, dtype=weight.dtype, device=weight.device)
        C.bcmt_embedding_forward(p, ids.contiguous(), _dense(weight), out)
    return out


def embedding_backward(ids, dout, V: int, scale: float = 1.0):
    """Gradient [V, D] of the table from dout [*ids.shape, D]."""
    _need(dout.shape[:-1] == ids.shape, f"dout must be [*ids.shape, D], not {tuple(dout.shape)}")
    _on(dout.device, ids=ids)
    D = dout.shape[-1]
    with torch.cuda.device(dout.device):
        p = _embedding_params(ids, V, D, _dtype(dout, "dout"), scale)
        dw = torch.empty(V, D, dtype=dout.dtype, device=dout.device)
        ws = _buffer(C.bcmt_embedding_workspace_size(p), dout.device)
        C.bcmt_embedding_backward(p, ids.contiguous(), _dense(dout), dw, ws)
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
        return None, embedding_backward(ids, dout, ctx.V, ctx.scale), None


def embedding(ids, weight, scale: float = 1.0):
    """Differentiable ``embedding_forward``."""
    return Embedding.apply(ids, weight, scale)


# --------------------------------------------------------------------- dropout
def _dropout_call(x, p, seed, offset, residual, step):
    _on(x.device, residual=residual, step=step)
    dt = _dtype(x, "x")
    if residual is not None:
        _need(residual.shape == x.shape and residual.dtype == x.dtype,
              f"residual must have x's shape and type: {tuple(residual.shape)} {residual.dtype}")
    if step is not None:
        _need(step.dtype == torch.int64 and step.numel() == 1, "step must be one int64")
    mask = (1 << 64) - 1
    with torch.cuda.device(x.device):
        x = _dense(x)
        y = torch.empty_like(x)
        prm = C.bcmt_dropout_params(x.numel(), dt, 0, p, seed & mask, offset & mask,
                                    None if step is None else step.data_ptr())
        C.bcmt_dropout(prm, x, _dense(residual), y)
    return y


def dropout_forward(x, p: float, seed: int, offset: int, residual=None, step=None):
    """``[residual +] keep * x / (1 - p)``, the mask a function of (seed, offset +
    step) and the element's index; step: an int64 on the device (for captured
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
        dx = dropout_backward(dy, *ctx.args, step=ctx.step) if ctx.needs_input_grad[0] else None
        return dx, None, None, None, dy if ctx.needs_input_grad[4] else None, None


def dropout(x, p: float, seed: int, offset: int, residual=None, step=None):
    """Differentiable ``dropout_forward``."""
    return Dropout.apply(x, p, seed, offset, residual, step)
