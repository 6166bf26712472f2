"""AdamW over many tensors in one launch, with states in 32 or in 8 bits.

``AdamWPlan`` is the bare call over a list of tensors, ``AdamW`` a
``torch.optim.Optimizer`` around it.  8-bit states are signed and unsigned bytes with
one float32 scale for every 256 consecutive elements of a tensor (``include/bcmt.h`` has
the code); ``adamw8_values`` gives the values that they stand for.  Everything runs on
the current CUDA stream; arguments that the library would misread raise ``ValueError``,
what it refuses raises ``bcmt.BCMTError``.
"""

from __future__ import annotations

import ctypes
from operator import attrgetter
from typing import Optional

import numpy as np
import torch
from torch.autograd.graph import increment_version

from . import bcmt as C
from .lm_ops import _address, _check, _current_device, _dense, _device, _dtype, _on_its_device, \
    _raw_stream

_F32 = torch.float32
BLOCK = 256   # elements that share a scale of 8-bit states
# what a step asks of every tensor, for map()
_SHAPE, _DTYPE = attrgetter("shape"), attrgetter("dtype")
_POINTER, _INDEX, _IS_DENSE = (torch.Tensor.data_ptr, torch.Tensor.get_device,
                               torch.Tensor.is_contiguous)
_P, _G, _M, _V, _W, _MS, _VS, _N = range(8)   # fields of bcmt_adamw_tensor


def _overlap(tensors):
    """Whether two of the (dense) tensors share memory."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())
                   for t in tensors if t.numel())
    return any(a[1] > b[0] for a, b in zip(spans, spans[1:]))


class AdamWPlan:
    """One AdamW step over the tensors of ``params`` (bf16 or fp32, all of one type, dense),
    which it updates in place with their states: m and v fp32 of the same shapes, or, with
    m_scales and v_scales, int8 and uint8 of as many elements with [ceil(n / 256)] fp32 scales.
    masters: fp32 values of bf16 params, which are then what is updated and params their
    rounding.  States start as zeros.  The plan holds the tensors, and reads their addresses
    at each step."""

    def __init__(self, params, m, v, *, masters=None, m_scales=None, v_scales=None):
        params, m, v = list(params), list(m), list(v)
        lists = [params, m, v]
        self.bits = 32 if m_scales is None and v_scales is None else 8
        if (m_scales is None) != (v_scales is None):
            raise ValueError("m_scales and v_scales belong together")
        self._columns = [_P, _M, _V]
        for t, column in ((masters, _W), (m_scales, _MS), (v_scales, _VS)):
            if t is not None:
                lists.append(list(t))
                self._columns.append(column)
        if any(len(t) != len(params) for t in lists):
            raise ValueError("params, states, masters and scales must be lists of one length")
        if not params:
            raise ValueError("params must have a tensor")
        if not all(isinstance(t, torch.Tensor) for x in lists for t in x):
            raise ValueError("params, states, masters and scales must be tensors")
        self.device = _device(params[0])
        self.dtype = params[0].dtype
        self._dt = _dtype(params[0], "params")
        if masters is not None and self.dtype == _F32:
            raise ValueError("float32 params have no masters")
        self._lists, self._all = lists, [t for x in lists for t in x]
        self._check()
        self._table = np.zeros((len(params), 8), dtype=np.int64)
        self._address = self._table.ctypes.data
        self._shapes = [p.shape for p in params]
        self._sizes = np.array([p.numel() for p in params], dtype=np.int64)
        self._at = None
        self._table[:, _N] = self._sizes
        self._holes = False

    def _check(self):
        dev = self.device
        for column, tensors in zip(self._columns, self._lists):
            name = ("params", "", "m", "v", "masters", "m_scales", "v_scales")[column]
            for p, t in zip(self._lists[0], tensors):
                shape, dtype = p.shape, self.dtype if column == _P else _F32
                if column in (_MS, _VS):
                    shape = (-(-p.numel() // BLOCK),)
                elif self.bits == 8 and column in (_M, _V):
                    shape, dtype = t.shape, torch.int8 if column == _M else torch.uint8
                    if t.numel() != p.numel():
                        raise ValueError(f"{name} must have {p.numel()} elements, not {t.numel()}")
                _check(t, name, shape, dtype, dev)
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be dense")
        if _overlap(self._all):
            raise ValueError("params, states, masters and scales must not share memory")

    def _refresh(self):
        at = list(map(_POINTER, self._all))
        if at != self._at:
            self._check()
            n = len(self._shapes)
            for i, column in enumerate(self._columns):
                self._table[:, column] = at[i * n:(i + 1) * n]
            self._at = at

    def _addresses(self, grads, dev):
        """(the gradients' addresses, 0 for None; copies that are to live until the launch)."""
        try:    # most often all are there, dense and right
            if (list(map(_SHAPE, grads)) == self._shapes and set(map(_DTYPE, grads)) == {self.dtype}
                    and set(map(_INDEX, grads)) == {dev.index}
                    and False not in map(_IS_DENSE, grads)):
                return list(map(_POINTER, grads)), None
        except (AttributeError, TypeError, RuntimeError):
            pass
        at, kept = [], []
        for g, shape in zip(grads, self._shapes):
            if g is None:
                at.append(0)
                continue
            if g.layout is not torch.strided:
                raise ValueError("grads must be dense tensors, not sparse ones")
            _check(g, "grads", shape, self.dtype, dev)
            if not g.is_contiguous():
                g = g.contiguous()
                kept.append(g)
            at.append(g.data_ptr())
        return at, kept

    @torch.no_grad()
    def step(self, grads, *, lr, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
             step, grad_scale: Optional[torch.Tensor] = None):
        """One step, the ``step``-th (from 1), with ``grads`` of the params' shapes and type
        (None: that tensor is left as it is).  step: an int, or one int64 on the device, and lr a
        number, or one float32 on the device, both then read when the kernel runs (captured
        graphs); grad_scale: one float32 on the device that the gradients are multiplied by."""
        dev = self.device
        if dev.index != _current_device():
            with torch.cuda.device(dev):
                return self.step(grads, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay,
                                 step=step, grad_scale=grad_scale)
        self._refresh()
        if len(grads) != len(self._shapes):
            raise ValueError(f"{len(self._shapes)} gradients are needed, not {len(grads)}")
        at, kept = self._addresses(grads, dev)
        table = self._table
        table[:, _G] = at
        holes = 0 in at
        if holes or self._holes:
            table[:, _N] = np.where(table[:, _G] != 0, self._sizes, 0)
            self._holes = holes
        step_ptr = lr_ptr = None
        if isinstance(step, torch.Tensor) and step.is_cuda:
            _one(step, "step", torch.int64, dev)
            step, step_ptr = 1, step.data_ptr()
        if isinstance(lr, torch.Tensor) and lr.is_cuda:
            _one(lr, "lr", _F32, dev)
            lr, lr_ptr = 0.0, lr.data_ptr()
        if grad_scale is not None:
            _one(grad_scale, "grad_scale", _F32, dev)
            grad_scale = grad_scale.data_ptr()
        p = C.bcmt_adamw_params(len(at), self._dt, self.bits, 0, int(step), float(lr), betas[0],
                                betas[1], eps, weight_decay, grad_scale, step_ptr, lr_ptr)
        C.check(C.LIB.bcmt_adamw_step(ctypes.byref(p), self._address, _raw_stream(dev.index)))
        # written through their addresses, which autograd cannot see
        increment_version([t for x in self._lists for t, g in zip(x, at) if g] if holes else self._all)


def _one(t, name, dtype, dev):
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.numel() != 1 or t.device != dev:
        raise ValueError(f"{name} must be one {dtype} on {dev}")


def _codes(t, name, dtype, dev):
    if t.dtype != dtype or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be dense {dtype} on {dev}")
    return _dense(t)


@_on_its_device
def adamw8_values(m, m_scale, v, v_scale):
    """The fp32 values (m, v) that 8-bit states stand for: m int8 and v uint8 of one shape,
    scales [ceil(n / 256)] fp32."""
    dev = _device(m)
    m, v = _codes(m, "m", torch.int8, dev), _codes(v, "v", torch.uint8, dev)
    if v.shape != m.shape:
        raise ValueError(f"v must be {tuple(m.shape)}, not {tuple(v.shape)}")
    blocks = (-(-m.numel() // BLOCK),)
    _check(m_scale, "m_scale", blocks, _F32, dev)
    _check(v_scale, "v_scale", blocks, _F32, dev)
    m_scale, v_scale = _dense(m_scale), _dense(v_scale)
    mo = torch.empty(m.shape, dtype=_F32, device=dev)
    vo = torch.empty(m.shape, dtype=_F32, device=dev)
    C.check(C.LIB.bcmt_adamw_values(m.data_ptr(), m_scale.data_ptr(), v.data_ptr(),
                                    v_scale.data_ptr(), mo.data_ptr(), vo.data_ptr(), m.numel(),
                                    _raw_stream(dev.index)))
    return mo, vo


def _options(group):
    """Refuses what would change the step in a group of torch's optimizers, and has no place here."""
    for name in ("maximize", "amsgrad", "differentiable"):
        if group.get(name):
            raise ValueError(f"this AdamW has no {name}")
    if not group.get("decoupled_weight_decay", True) and group["weight_decay"] != 0:
        raise ValueError("decoupled_weight_decay=False: the weight decay of AdamW is decoupled")
    if group.get("bits", 32) not in (32, 8):
        raise ValueError(f"bits must be 32 or 8, not {group['bits']}")


def _states(bits):
    """Names and types of a parameter's states."""
    if bits == 8:
        return {"exp_avg": torch.int8, "exp_avg_sq": torch.uint8, "exp_avg_scale": _F32,
                "exp_avg_sq_scale": _F32}
    return {"exp_avg": _F32, "exp_avg_sq": _F32}


def _capturing(p):
    """Whether what runs on p's device now goes into a graph."""
    if not p.is_cuda:
        return False
    if p.get_device() != _current_device():
        with torch.cuda.device(p.device):
            return torch.cuda.is_current_stream_capturing()
    return torch.cuda.is_current_stream_capturing()


def _has_master(group, p):
    return group["masters"] and p.dtype != _F32


def _check_file(group, states):
    """Refuses a file's states that are not those of its (completed) group."""
    names = _states(group["bits"])
    for k in group["params"]:
        s = states.get(k)
        if not s:
            continue
        lacking = [n for n in (*names, "step") if n not in s]
        # floats of another width are taken, as torch's files of bf16 parameters have them
        lacking += [f"{n} as {t}" for n, t in names.items()
                    if n in s and s[n].dtype != t and not (t.is_floating_point and s[n].is_floating_point())]
        if lacking:
            raise ValueError(f"parameter {k} of the file has no {', '.join(lacking)}: the group's states "
                             f"are in {group['bits']} bits")


class AdamW(torch.optim.Optimizer):
    """AdamW with every tensor of a parameter group in one launch.

    bits: 32, or 8 for states in 8 bits; masters: float32 values of bf16 parameters are kept
    and updated.  capturable: the count of steps is kept on the device, so that a captured
    ``step`` goes on counting at each replay (the group then counts as one, but for parameters
    that were behind the others in a file); with an lr that is a float32 on the device, the rate
    can change between replays too.  A parameter's first step, which begins its states, is to be
    outside of the capture; captures that hold one, or are not capturable, raise RuntimeError.
    ``step`` takes a grad_scale (one float32 on the device, as from clipping by the norm).

    Files of torch.optim.AdamW load where bits is 32; masters (then begun from the parameters) and
    capturable=True stay as they are.  Groups and files that ask for a step of another kind
    (maximize, amsgrad, differentiable, a weight decay that is not decoupled) or lack the group's
    states raise ValueError."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 1e-2, *, bits: int = 32, masters: bool = False,
                 capturable: bool = False):
        _options(dict(bits=bits))
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay,
                                      bits=bits, masters=masters, capturable=capturable))
        self._plans = {}

    def __setstate__(self, state):   # a copy, or groups out of a file
        super().__setstate__(state)
        self._plans = {}
        for group in self.param_groups:
            for k in ("bits", "masters", "capturable"):
                group.setdefault(k, self.defaults.get(k))

    def add_param_group(self, param_group):
        if isinstance(param_group, dict):   # (torch refuses anything else)
            _options({**self.defaults, **param_group})
        super().add_param_group(param_group)

    def _init(self, p, group, moved):
        """What p's state lacks: everything at its first step, a master that a file had none of, and
        the count where the group has it now (moved: those of this step, by device and value)."""
        s = self.state[p]
        capturable = bool(group["capturable"])
        missing = "master" not in s and _has_master(group, p)
        move = bool(s) and isinstance(s["step"], torch.Tensor) is not capturable
        if (missing or move or not s) and _capturing(p):
            raise RuntimeError("a parameter's first step begins its states, and would at each replay: "
                               "take it before the capture")
        if move:
            n = int(s["step"])
            s["step"] = n if not capturable else \
                moved.setdefault((p.device, n), torch.tensor(n, device=p.device))
        if not s:
            flat = torch.preserve_format if p.is_contiguous() else torch.contiguous_format
            if group["bits"] == 8:
                blocks = -(-p.numel() // BLOCK)
                s["exp_avg"] = torch.zeros(p.shape, dtype=torch.int8, device=p.device)
                s["exp_avg_sq"] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device)
                s["exp_avg_scale"] = torch.zeros(blocks, dtype=_F32, device=p.device)
                s["exp_avg_sq_scale"] = torch.zeros(blocks, dtype=_F32, device=p.device)
            else:
                s["exp_avg"] = torch.zeros_like(p, dtype=_F32, memory_format=flat)
                s["exp_avg_sq"] = torch.zeros_like(p, dtype=_F32, memory_format=flat)
            s["step"] = self._count(group, p.device) if capturable else 0
        if missing:
            s["master"] = p.detach().to(_F32)

    def _count(self, group, device):   # on the device: one there for the group
        for p in group["params"]:
            count = self.state[p].get("step") if p in self.state and p.device == device else None
            if isinstance(count, torch.Tensor):
                return count
        return torch.zeros((), dtype=torch.int64, device=device)

    def _plan(self, key, group, params, states):
        names = list(_states(group["bits"]))
        names += ["master"] if _has_master(group, params[0]) else []
        ids = [id(p) for p in params] + [id(s[k]) for s in states for k in names]
        plan = self._plans.get(key)
        if plan is None or plan[0] != ids:
            of = {k: [s[k] for s in states] for k in names}
            plan = (ids, AdamWPlan(params, of["exp_avg"], of["exp_avg_sq"], masters=of.get("master"),
                                   m_scales=of.get("exp_avg_scale"),
                                   v_scales=of.get("exp_avg_sq_scale")))
            self._plans[key] = plan
        return plan[1]

    @torch.no_grad()
    def step(self, closure=None, *, grad_scale: Optional[torch.Tensor] = None):
        loss = None
        for group in self.param_groups:
            _options(group)
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for i, group in enumerate(self.param_groups):
            kinds, moved = {}, {}
            capturable, masters = bool(group["capturable"]), group["masters"]
            for p in group["params"]:
                if p.grad is None:
                    continue
                if not kinds and not capturable and _capturing(p):
                    raise RuntimeError("a captured step would repeat its count: capturable=True keeps "
                                       "the count on the device")
                s = self.state[p]
                if (not s or isinstance(s["step"], torch.Tensor) is not capturable
                        or (masters and "master" not in s)):
                    self._init(p, group, moved)
                kind = (p.dtype, p.device, id(s["step"]) if capturable else None)
                if kind not in kinds:
                    kinds[kind] = [], []
                params, states = kinds[kind]
                params.append(p)
                states.append(s)
            how = dict(lr=group["lr"], betas=group["betas"], eps=group["eps"],
                       weight_decay=group["weight_decay"], grad_scale=grad_scale)
            counted = set()
            for kind, (params, states) in kinds.items():
                plan = self._plan((i, kind), group, params, states)
                grads = [p.grad for p in params]
                if capturable:
                    count = states[0]["step"]
                    first = id(count) not in counted
                    if first:
                        count += 1
                    try:
                        plan.step(grads, step=count, **how)
                    except Exception:   # a refused step does not count
                        if first:
                            count -= 1
                        raise
                    counted.add(id(count))
                    continue
                steps = [s["step"] + 1 for s in states]
                each = sorted(set(steps))
                for n in each:   # parameters that had no gradient in some steps are behind
                    plan.step(grads if len(each) == 1 else
                              [g if k == n else None for g, k in zip(grads, steps)], step=n, **how)
                    for s, k in zip(states, steps):
                        if k == n:
                            s["step"] = n
        return loss

    @torch.no_grad()
    def load_state_dict(self, state_dict):
        groups = list(state_dict["param_groups"])
        for i, (saved, group) in enumerate(zip(groups, self.param_groups)):
            if "bits" not in saved:   # of another optimizer: what it does not know stays
                groups[i] = saved = {**saved, "bits": group["bits"], "masters": group["masters"],
                                     "capturable": group["capturable"] or saved.get("capturable", False)}
            _options(saved)
            _check_file(saved, state_dict["state"])
        state_dict = {**state_dict, "param_groups": groups}
        super().load_state_dict(state_dict)
        # the states in their own types (the base class gives them the parameters'): all floats are
        # float32, moments that torch kept in bf16 too
        for group, saved in zip(self.param_groups, state_dict["param_groups"]):
            count = {}   # on the device: one there for all parameters of the same count
            for p, k in zip(group["params"], saved["params"]):
                for name, x in state_dict["state"].get(k, {}).items():
                    if name == "step":
                        x = int(x)
                        if group["capturable"]:
                            x = count.setdefault((p.device, x), torch.tensor(x, device=p.device))
                    elif isinstance(x, torch.Tensor):
                        x = x.detach().to(p.device, _F32 if x.is_floating_point() else x.dtype, copy=True)
                    self.state[p][name] = x
        self._plans.clear()
