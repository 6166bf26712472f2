"""The end of a block of the language model fused with the norm before the next:
``h = residual_scale * x + gate * post(branch)``, ``n = pre(h)``.

Marshalling only, as in ``lm_ops``: each call runs the library's kernels
(``include/bcmt.h``) on the current CUDA stream.  ``residual_norm`` is
differentiable (once); ``residual_norm_forward`` and ``residual_norm_backward`` are
the bare calls.  Arguments that the library would misread raise ``ValueError``;
what the library refuses raises ``bcmt.BCMTError``.
"""

from __future__ import annotations

import ctypes
import functools
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import bcmt as C
from .lm_ops import (_address, _buffer, _check, _current_device, _dense, _device, _dtype, _number,
                     _on_its_device, _raw_stream)

KINDS = ("layer", "rms")
_ALL = (True,) * 7   # gradients


@functools.lru_cache(maxsize=4096)
def _plan(rows, D, dt, wt, rms, gates, alpha, eps, post):
    """(parameters by reference, bytes of the backward's workspace)."""
    p = C.bcmt_norm_params(rows, D, dt, wt, rms, gates, 0, alpha, eps)
    return ctypes.byref(p), C.bcmt_residual_norm_workspace_size(p, post)


def _gates(gate, shape) -> int:
    """Rows of a gate that broadcasts to ``shape``: [D], or the leading dimensions of
    ``shape``, ones, and D, so that consecutive rows share one."""
    g = tuple(gate.shape)
    if g == tuple(shape):
        return gate.numel() // shape[-1] if shape[-1] else 0
    full = (1,) * (len(shape) - len(g)) + g
    i = len(full) - 1
    while i > 0 and full[i - 1] == 1:
        i -= 1
    if len(g) < 1 or len(full) != len(shape) or full[-1] != shape[-1] or full[:i] != tuple(shape[:i]):
        raise ValueError(f"gate must be [D] or leading dimensions of {tuple(shape)}, ones and D, "
                         f"not {g}")
    n = 1
    for d in full[:i]:
        n *= d
    return n


def _same(t, name, shape, dtype, dev):
    """``_check`` for a tensor on a CUDA device, quicker where it is right."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev.index:
        _check(t, name, shape, dtype, dev)


def _arguments(branch, weight, bias, post_weight, post_bias, gate, kind):
    """(device, shape, dtype, weights' dtype, rows of the gate), after the checks of what both
    passes take."""
    dev, shape, dtype = _device(branch), branch.shape, weight.dtype
    dt = _dtype(branch, "branch")
    if not shape:
        raise ValueError("branch must be [..., D]")
    if kind not in KINDS:
        raise ValueError(f"kind must be one of {KINDS}, not {kind!r}")
    wt = _dtype(weight, "weight")
    vector = shape[-1:]
    _same(weight, "weight", vector, dtype, dev)
    if bias is not None:
        _same(bias, "bias", vector, dtype, dev)
    if post_weight is not None:
        _same(post_weight, "post_weight", vector, dtype, dev)
    if post_bias is not None:
        _same(post_bias, "post_bias", vector, dtype, dev)
        if post_weight is None:
            raise ValueError("post_bias without post_weight")
    gates = 0
    if gate is not None:
        gates = _gates(gate, shape)
        _same(gate, "gate", gate.shape, branch.dtype, dev)
    return dev, shape, dt, wt, gates


@_on_its_device
def residual_norm_forward(branch, x, weight, bias=None, *, post_weight=None, post_bias=None,
                          gate=None, residual_scale: float = 1.0, kind: str = "layer",
                          eps: float = 1e-5):
    """(h, n) of ``h = residual_scale * x + gate * post(branch)``, ``n = pre(h)``.

    branch, x [..., D] (bf16 or fp32; 1 <= D <= 8192); weight, bias [D] of the pre norm and
    post_weight, post_bias [D] of the post norm, all of one type (bf16 or fp32; no
    post_weight: no post norm); kind: both are layer norms ("layer") or root-mean-square
    norms ("rms").  gate: [D], or one for every leading index ([B, 1, D] for branch
    [B, T, D]), or of branch's shape; default 1."""
    dev, shape, dt, wt, gates = _arguments(branch, weight, bias, post_weight, post_bias, gate, kind)
    _same(x, "x", shape, branch.dtype, dev)
    D = shape[-1]
    rows = branch.numel() // D if D else 0
    p, _ = _plan(rows, D, dt, wt, int(kind == "rms"), gates, _number(residual_scale, "residual_scale"),
                 _number(eps, "eps"), post_weight is not None)
    branch, x, weight, bias = _dense(branch), _dense(x), _dense(weight), _dense(bias)
    post_weight, post_bias, gate = _dense(post_weight), _dense(post_bias), _dense(gate)
    h, n = torch.empty_like(branch), torch.empty_like(branch)
    C.check(C.LIB.bcmt_residual_norm_forward(
        p, branch.data_ptr(), x.data_ptr(), weight.data_ptr(), _address(bias),
        _address(post_weight), _address(post_bias), _address(gate), h.data_ptr(), n.data_ptr(),
        _raw_stream(dev.index)))
    return h, n


def residual_norm_backward(dh, dn, branch, h, weight, bias=None, *, post_weight=None,
                           post_bias=None, gate=None, residual_scale: float = 1.0,
                           kind: str = "layer", eps: float = 1e-5, wanted=_ALL):
    """(dbranch, dx, dweight, dbias, dpost_weight, dpost_bias, dgate) from the forward's
    arguments, its h and the gradients dh (None: zero) and dn of its results; None for what
    was not given.  dbranch and dx are one tensor where they are equal (no post norm, no gate,
    residual_scale 1).  wanted: which of the seven to compute; the others are None, but for
    dbranch, which comes anyway."""
    # (dh may be None: the device is that of branch)
    if isinstance(branch, torch.Tensor) and branch.is_cuda and branch.get_device() != _current_device():
        with torch.cuda.device(branch.device):
            return residual_norm_backward(
                dh, dn, branch, h, weight, bias, post_weight=post_weight, post_bias=post_bias,
                gate=gate, residual_scale=residual_scale, kind=kind, eps=eps, wanted=wanted)
    dev, shape, dt, wt, gates = _arguments(branch, weight, bias, post_weight, post_bias, gate, kind)
    dtype = branch.dtype
    _same(dn, "dn", shape, dtype, dev)
    _same(h, "h", shape, dtype, dev)
    if dh is not None:
        _same(dh, "dh", shape, dtype, dev)
    D = shape[-1]
    rows = branch.numel() // D if D else 0
    alpha = _number(residual_scale, "residual_scale")
    p, nbytes = _plan(rows, D, dt, wt, int(kind == "rms"), gates, alpha, _number(eps, "eps"),
                      post_weight is not None)
    dh, dn, branch, h = _dense(dh), _dense(dn), _dense(branch), _dense(h)
    weight, post_weight, post_bias = _dense(weight), _dense(post_weight), _dense(post_bias)
    one = post_weight is None and gate is None and alpha == 1.0
    gate = _dense(gate)
    like = torch.empty_like
    _, want_x, want_w, want_b, want_pw, want_pb, want_gate = wanted
    dbranch = like(branch)
    dx = None if one or not want_x else like(branch)
    dw = like(weight) if want_w else None
    db = None if bias is None or not want_b else like(weight)
    dpw = None if post_weight is None or not want_pw else like(weight)
    dpb = None if post_bias is None or not want_pb else like(weight)
    dgate = None if gate is None or not want_gate else like(gate)
    ws = _buffer(max(256, nbytes), dev)
    C.check(C.LIB.bcmt_residual_norm_backward(
        p, _address(dh), dn.data_ptr(), branch.data_ptr(), h.data_ptr(), weight.data_ptr(),
        _address(post_weight), _address(post_bias), _address(gate), dbranch.data_ptr(),
        _address(dx), _address(dw), _address(db), _address(dpw), _address(dpb), _address(dgate),
        ws.data_ptr(), _raw_stream(dev.index)))
    return dbranch, dbranch if one and want_x else dx, dw, db, dpw, dpb, dgate


class ResidualNorm(torch.autograd.Function):
    """(h, n) with branch, x, the norms' weights and the gate as differentiable inputs."""

    @staticmethod
    def forward(ctx, branch, x, weight, bias, post_weight, post_bias, gate, alpha, kind, eps):
        h, n = residual_norm_forward(branch, x, weight, bias, post_weight=post_weight,
                                     post_bias=post_bias, gate=gate, residual_scale=alpha,
                                     kind=kind, eps=eps)
        ctx.save_for_backward(branch, h, weight, bias, post_weight, post_bias, gate)
        ctx.args = (alpha, kind, eps)
        ctx.set_materialize_grads(False)
        return h, n

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dn):
        branch, h, weight, bias, post_weight, post_bias, gate = ctx.saved_tensors
        alpha, kind, eps = ctx.args
        if dh is None and dn is None:
            return (None,) * 10
        if dn is None:
            dn = torch.zeros_like(h)
        return residual_norm_backward(
            dh, dn, branch, h, weight, bias, post_weight=post_weight, post_bias=post_bias,
            gate=gate, residual_scale=alpha, kind=kind, eps=eps,
            wanted=ctx.needs_input_grad[:7]) + (None,) * 3


def residual_norm(branch, x, weight, bias=None, *, post_weight=None, post_bias=None, gate=None,
                  residual_scale: float = 1.0, kind: str = "layer", eps: float = 1e-5):
    """Differentiable ``residual_norm_forward``."""
    return ResidualNorm.apply(branch, x, weight, bias, post_weight, post_bias, gate,
                              _number(residual_scale, "residual_scale"), kind, _number(eps, "eps"))
