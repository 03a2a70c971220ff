"""The server's update of a model that lies in many tensors: the global norm of the gradient and the AdamW step, each one
pass over all of them.

The handles hold what the calls need on the device (the plan of the tensors' chunks, states, partial sums) and issue
them; all arithmetic runs in the HIP kernels (``co3_grad_norm``, ``co3_adamw``, ``co3_adamw8``).  Calls are issued on the
current stream of the tensors' device and return without waiting.  Calls of one handle, replays of graphs that hold them
among these, share its workspaces: they must not run at the same time.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import operator
from typing import List, Optional, Sequence, Union

import numpy as np
import torch

from . import binding as B

try:
    from ._tensors import look as _look, same as _same
except ImportError as e:
    raise ImportError("the host module _tensors.so is not built, or for another torch; run "
                      "`python -c 'import __graft_entry__ as g; g.build()'`") from e

PerTensor = Union[float, Sequence[float]]

# the handle of a device's current stream without the object around it (0.1 us against 1.8)
_raw_stream = torch._C._cuda_getCurrentRawStream


def _per_tensor(x: PerTensor, T: int, what: str) -> List[float]:
    values = [float(x)] * T if isinstance(x, (int, float)) else [float(v) for v in x]
    if len(values) != T:
        raise ValueError(f"{what}: one value per tensor is needed ({T}), got {len(values)}")
    if not all(v >= 0.0 and math.isfinite(v) for v in values):
        raise ValueError(f"{what} must be finite and not negative")
    return values


def _check_scale(grad_scale: float):
    if not 2.0 ** -126 <= grad_scale <= 2.0 ** 127:
        raise ValueError("grad_scale must be between 2^-126 and 2^127")


def _check_tensors(tensors: Sequence[torch.Tensor], what: str):
    if not tensors:
        raise ValueError(f"no {what}")
    if not all(isinstance(t, torch.Tensor) and t.is_cuda for t in tensors):
        raise ValueError(f"{what}: CUDA tensors are needed")
    dtype, device = tensors[0].dtype, tensors[0].get_device()
    if dtype not in B.TYPE_OF or not all(t.dtype is dtype for t in tensors):
        raise ValueError(f"{what}: all of one type out of float32, bfloat16 and float16 (MixedAdamW takes several)")
    if not all(t.get_device() == device for t in tensors):
        raise ValueError(f"{what}: all on one device")
    if not all(t.is_contiguous() for t in tensors):
        raise ValueError(f"{what}: contiguous tensors are needed")


def _overlapping(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor]) -> bool:
    """Whether a parameter shares memory with another one or with a gradient."""
    spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), kind) for kind, ts in enumerate((params, grads)) for t in ts
                   if t.numel())
    end_any = end_param = 0
    for lo, hi, kind in spans:
        if lo < end_param or (kind == 0 and lo < end_any):
            return True
        end_any = max(end_any, hi)
        end_param = max(end_param, hi) if kind == 0 else end_param
    return False


class _Table:
    """Plan of a list of tensors on their device.  The tensors are looked at before every use (address, elements, type,
    contiguity), and a new plan is made when one has moved or is of another type."""

    def __init__(self, params: Optional[Sequence[torch.Tensor]], grads: Sequence[torch.Tensor], state_bits: int,
                 lr_scales: PerTensor = 1.0, weight_decays: PerTensor = 0.0):
        self.params = None if params is None else list(params)
        self.state_bits = state_bits
        self._take(grads)
        T = len(self.grads)
        self.device = self.grads[0].device
        self.lr_scales, self.weight_decays = _per_tensor(lr_scales, T, "lr_scales"), _per_tensor(weight_decays, T, "weight_decay")
        self._captured = []                      # plans and learning rates that a captured graph goes on reading
        self.lr = None                           # the learning rate and its memory, where it lies on the device
        self.masters = False
        self.also = []                           # memory of the handle that its launches use, made on the stream that is current now
        with torch.cuda.device(self.device):
            self._streams = {_raw_stream(self.device.index)}
        self._make()

    def _take(self, grads: Sequence[torch.Tensor]):
        grads = list(grads)
        self._check(grads)
        self.sizes = [g.numel() for g in grads]
        self.grads = grads

    def _check(self, grads: Sequence[torch.Tensor]):
        _check_tensors(grads, "gradients")
        sizes = getattr(self, "sizes", None) or [p.numel() for p in self.params or grads]
        if self.params is not None:
            _check_tensors(self.params, "parameters")
            if sizes != [p.numel() for p in self.params]:
                raise ValueError("parameters: as many elements as before")
            if getattr(self, "masters", False) and self.params[0].dtype == torch.float32:
                raise ValueError("float32 parameters are their own masters")
            if grads[0].device != self.params[0].device:
                raise ValueError("gradients: on the parameters' device")
        if sizes != [g.numel() for g in grads]:
            raise ValueError("gradients: one per parameter, with as many elements")

    def _make(self):
        T = len(self.grads)
        watched = self.grads + (self.params or [])
        seen, at = _look(watched), [t.data_ptr() for t in watched]
        table = np.zeros(T, dtype=[("param", "u8"), ("grad", "u8"), ("n", "i8"), ("lr_scale", "f4"), ("weight_decay", "f4")])
        if self.params is not None:
            table["param"] = at[T:]
        table["grad"], table["n"] = at[:T], self.sizes
        table["lr_scale"], table["weight_decay"] = self.lr_scales, self.weight_decays
        rows = (B.StepTensor * T).from_buffer(table)
        layout = B.step_layout_of(rows, B.TYPE_NONE if self.params is None else B.TYPE_OF[self.params[0].dtype],
                                  B.TYPE_OF[self.grads[0].dtype], self.state_bits)
        try:
            host = B.step_plan(rows, layout)
        except B.Co3Error as e:
            raise ValueError("a parameter shares memory with another one or with a gradient") from e
        with torch.cuda.device(self.device):
            self.plan = host.to(self.device)
            # the streams that all of the memory is known to: the plan to this one alone, `also` to those it was known to before
            raw = _raw_stream(self.device.index)
            self._streams = {raw} & self._streams
        self.layout, self.layout_ref, self.plan_ptr = layout, C.byref(layout), C.c_void_p(self.plan.data_ptr())
        self._watched, self._seen = watched, seen                # what the plan is for

    def now(self):
        """Gradients and plan as they are, for ``back``."""
        return self.grads, self.plan, self._streams, self.layout, self.layout_ref, self.plan_ptr, self._watched, self._seen

    def back(self, was):
        self.grads, self.plan, self._streams, self.layout, self.layout_ref, self.plan_ptr, self._watched, self._seen = was

    def ready(self, grads: Optional[Sequence[torch.Tensor]], capturable: bool = True) -> C.c_void_p:
        """The plan is that of the tensors as they lie now; returns the current stream of their device, which is the current one."""
        capturing = torch.cuda.is_current_stream_capturing()
        if capturing and not capturable:
            raise RuntimeError("a captured step needs device_steps=True")
        was = self.grads
        if grads is not None:
            self._take(grads)
            self._watched = self.grads + (self.params or [])
        if not _same(self._watched, self._seen):
            try:
                if capturing:
                    raise RuntimeError("a tensor has moved or changed since the last call: call once before the capture")
                if grads is None:
                    self._check(self.grads)
                self._make()
            except Exception:
                self.grads = was                                 # refused gradients are not kept
                self._watched = was + (self.params or [])
                raise
        raw = _raw_stream(self.device.index)
        if capturing:
            if not any(plan is self.plan and lr is self.lr for plan, lr in self._captured):
                self._captured.append((self.plan, self.lr))
        elif raw not in self._streams:
            self._streams.add(raw)
            for t in [self.plan] + self.also + ([] if self.lr is None else [self.lr[0]]):
                t.record_stream(torch.cuda.current_stream(self.device))
        return C.c_void_p(raw)


def _on_device(call):
    """Launches of a handle go to its tensors' device, whichever is current."""
    @functools.wraps(call)
    def there(self, grads=None):
        device = self._table.device
        if torch.cuda.current_device() == device.index:
            return call(self, grads)
        with torch.cuda.device(device):
            return call(self, grads)
    return there


class GradNorm:
    """Global L2 norm of gradients that lie in many tensors, with the factor that clips it.

    ``compute()`` returns a float32 tensor of two on the device, (norm, factor): norm = grad_scale * sqrt(sum g^2),
    factor = grad_scale * min(1, max_norm / (norm + 1e-6)), or -1 where a gradient is not finite (a norm beyond float32 alone is
    infinite with its factor right).  The tensor is the handle's: the next call overwrites it."""

    def __init__(self, grads: Sequence[torch.Tensor], max_norm: float = math.inf, grad_scale: float = 1.0):
        if not max_norm > 0.0:
            raise ValueError("max_norm must be positive")
        _check_scale(grad_scale)
        self.max_norm, self.grad_scale = float(max_norm), float(grad_scale)
        self._table = _Table(None, grads, 0)
        dev = self._table.device
        self._out = torch.zeros(2, dtype=torch.float32, device=dev)
        self._partials = torch.zeros(self._table.layout.partials, dtype=torch.float64, device=dev)
        self._ptrs = C.c_void_p(self._out.data_ptr()), C.c_void_p(self._partials.data_ptr())
        self._table.also = [self._out, self._partials]
        torch.cuda.current_stream(dev).synchronize()       # cleared, for whichever stream comes first

    @_on_device
    def compute(self, grads: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
        """``grads``: None, or tensors of the same sizes to take instead, from now on."""
        t = self._table
        stream = t.ready(grads)
        B._chk(B._lib.co3_grad_norm(t.layout_ref, t.plan_ptr, self.grad_scale, self.max_norm, *self._ptrs, stream), "co3_grad_norm")
        return self._out


class AdamW:
    """AdamW over many tensors at once (the formulas: ``include/co3.h``).

    params, grads   tensors of one type each (float32, bfloat16, float16), contiguous, on one device; written and read in place
    lr              a float, or a float32 tensor of one element on the device (read at every step, also of a replayed graph)
    weight_decay, lr_scales   one value, or one per tensor
    state_bits      32: ``m``, ``v`` float32.  8: ``m``, ``r`` float8_e4m3fn with ``m_scale``, ``r_scale`` float8_e8m0fnu per 256 elements
                    (r = sqrt(v)), rounded at random by a hash of ``seed``, the step and the place
    master          16-bit parameters: float32 values kept in ``master``, taken from the parameters at the start
    max_norm        None, or the global norm beyond which the gradients are scaled down; a step with a gradient that is not finite
                    changes nothing and does not count (``skipped``)
    grad_scale      multiplies every gradient (1 / loss scale, say)
    device_steps    the device counts the steps, which a captured step needs (always so with max_norm or a tensor ``lr``)

    The state arrays hold the tensors one behind another: packed with 32 bits, each from a multiple of 256 on with 8.  They stay the
    handle's: a program copies into them.  A graph that holds a captured step needs the handle alive, and the parameters and
    gradients that it was captured with; a learning rate on the device the handle keeps for it.
    """

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], lr: Union[float, torch.Tensor] = 1e-3,
                 betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: PerTensor = 0.01, lr_scales: PerTensor = 1.0,
                 state_bits: int = 32, master: bool = False, max_norm: Optional[float] = None, grad_scale: float = 1.0, seed: int = 0,
                 device_steps: bool = False):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        if not all(0.0 <= b < 1.0 for b in betas):
            raise ValueError("betas must be in [0, 1)")
        if not (C.c_float(eps).value >= 2.0 ** -126 and math.isfinite(eps)):
            raise ValueError("eps must be finite and at least 2^-126")
        if max_norm is not None and not max_norm > 0.0:
            raise ValueError("max_norm must be positive")
        _check_scale(grad_scale)
        self._table = t = _Table(params, grads, state_bits, lr_scales, weight_decay)
        if master and t.params[0].dtype == torch.float32:
            raise ValueError("float32 parameters are their own masters")
        self.state_bits, self.max_norm = state_bits, max_norm
        self._args = B.AdamwArgs(0.0, betas[0], betas[1], eps, grad_scale, math.inf if max_norm is None else max_norm, 0,
                                 seed & 0xFFFFFFFFFFFFFFFF)
        self._args_ref = C.byref(self._args)
        z = dict(device=t.device)
        n, blocks = t.layout.elems, t.layout.blocks
        if state_bits == 32:
            self.m, self.v = (torch.zeros(n, dtype=torch.float32, **z) for _ in range(2))
            states = (self.m, self.v)
        else:
            self.m, self.r = (torch.zeros(n, dtype=torch.uint8, **z).view(torch.float8_e4m3fn) for _ in range(2))
            self.m_scale, self.r_scale = (torch.zeros(blocks, dtype=torch.uint8, **z).view(torch.float8_e8m0fnu) for _ in range(2))
            states = (self.m, self.m_scale, self.r, self.r_scale)
        self.master = None
        if master:
            self.master = torch.zeros(n, dtype=torch.float32, **z)
            t.masters = True
            self.take_masters()
        # an array of no elements has no address: any will do, none is read
        self._state_ptrs = [C.c_void_p(s.data_ptr() or t.plan.data_ptr()) for s in states]
        self._master_ptr = None if self.master is None else C.c_void_p(self.master.data_ptr() or t.plan.data_ptr())
        self._step_fn, self._clipped_fn = ((B._lib.co3_adamw, B._lib.co3_adamw_clipped) if state_bits == 32 else
                                           (B._lib.co3_adamw8, B._lib.co3_adamw8_clipped))
        self._t = 0
        self._dev = torch.zeros(B.STEP_STATE_BYTES // 8, dtype=torch.int64, **z)
        self._dev_ptr = C.c_void_p(self._dev.data_ptr())
        self.norm = self._dev.view(torch.float32)[4:6]        # (norm, factor) of the last step that took a norm
        self._partials = torch.zeros(t.layout.partials if max_norm is not None else 1, dtype=torch.float64, **z)
        self._partials_ptr = C.c_void_p(self._partials.data_ptr())
        self._device_steps = device_steps or max_norm is not None
        self._lr_seen = None
        self.lr = lr
        t.also = [self._dev, self._partials, *self._named().values()]
        torch.cuda.current_stream(t.device).synchronize()      # cleared, for whichever stream comes first

    # ---- what a program sets and reads
    @property
    def lr(self):
        return self._lr

    @lr.setter
    def lr(self, lr):
        if isinstance(lr, torch.Tensor):
            if lr.dtype != torch.float32 or lr.numel() != 1 or lr.device != self._table.device:
                raise ValueError("lr: a float32 tensor of one element on the parameters' device")
            if not self._device_steps:              # the device counts from here on
                if torch.cuda.is_current_stream_capturing():        # and would again at every replay
                    raise RuntimeError("lr as a tensor inside a capture needs device_steps=True")
                self._dev[0] = self._t
                self._device_steps = True
            self._args.lr = 0.0
            seen = _look([lr])
            if seen != self._lr_seen:
                self._lr_seen, self._lr_ptr = seen, C.c_void_p(lr.data_ptr())
                self._table.lr, self._table._streams = (lr, lr.untyped_storage()), set()      # known to no stream yet
        elif not (lr >= 0.0 and math.isfinite(lr)):
            raise ValueError("lr must be finite and not negative")
        else:
            self._args.lr = float(lr)
            self._lr_seen = self._lr_ptr = self._table.lr = None
        self._lr = lr

    def _look_at_lr(self):
        if self._lr_seen is not None and not _same([self._lr], self._lr_seen):
            self.lr = self._lr

    @property
    def t(self) -> int:
        """Number of steps taken (waits for the device where that counts them)."""
        return int(self._dev[0].item()) if self._device_steps else self._t

    @t.setter
    def t(self, t: int):
        if t < 0:
            raise ValueError("t must not be negative")
        self._t = int(t)
        self._dev[0] = int(t)

    @property
    def skipped(self) -> int:
        """Steps left out because their norm was not finite (waits for the device)."""
        return int(self._dev[1].item())

    def _views(self, flat: torch.Tensor) -> List[torch.Tensor]:
        unit, sizes = B.STEP_BLOCK if self.state_bits == 8 else 1, self._table.sizes
        parts = flat.split([(n + unit - 1) // unit * unit for n in sizes])
        if unit > 1:
            parts = [x[:n] for x, n in zip(parts, sizes)]
        return [x if p.dim() == 1 else x.view(p.shape) for x, p in zip(parts, self._table.params)]

    def take_masters(self):
        """Masters as the parameters are now (after the parameters were loaded from elsewhere)."""
        if self.master is not None:
            torch._foreach_copy_(self._views(self.master), [p.detach() for p in self._table.params])

    def moments(self):
        """(m, v) of every tensor as float32 copies, whatever the states are kept in."""
        if self.state_bits == 32:
            m, v = self.m.clone(), self.v.clone()
        else:
            wide = lambda x, s: (x.float().view(-1, B.STEP_BLOCK) * s.float()[:, None]).view(-1)  # noqa: E731
            m, v = wide(self.m, self.m_scale), wide(self.r, self.r_scale).square()
        return list(zip(self._views(m), self._views(v)))

    def _named(self):
        names = ("m", "v") if self.state_bits == 32 else ("m", "m_scale", "r", "r_scale")
        out = {k: getattr(self, k) for k in names}
        if self.master is not None:
            out["master"] = self.master
        return out

    def state_dict(self) -> dict:
        return {"t": self.t, "skipped": self.skipped, "seed": int(self._args.seed), **{k: v.clone() for k, v in self._named().items()}}

    def _check_state(self, d: dict):
        if not isinstance(d, dict):
            raise ValueError("state_dict: a dict is needed")
        for k, v in self._named().items():
            if not isinstance(d.get(k), torch.Tensor) or d[k].dtype != v.dtype or d[k].shape != v.shape:
                raise ValueError(f"state_dict: {k} is missing or of another type or size")
        for k in ("t", "skipped", "seed"):
            if not hasattr(d.get(k), "__index__") or operator.index(d[k]) < 0:
                raise ValueError(f"state_dict: {k} is missing or not a whole number from 0")

    def load_state_dict(self, d: dict):
        """All of a state, or, where some of it is missing or does not fit, nothing (ValueError)."""
        self._check_state(d)
        for k, v in self._named().items():
            v.copy_(d[k])
        self._args.seed = operator.index(d["seed"])
        self.t = d["t"]
        self._dev[1] = d["skipped"]

    # ---- the step
    @_on_device
    def step(self, grads: Optional[Sequence[torch.Tensor]] = None):
        """One step on every tensor.  ``grads``: None, or tensors of the same sizes to take instead, from now on."""
        t = self._table
        self._look_at_lr()
        stream = t.ready(grads, self._device_steps)
        if self.max_norm is not None:
            B._chk(self._clipped_fn(t.layout_ref, t.plan_ptr, self._master_ptr, *self._state_ptrs, self._args_ref, self._lr_ptr,
                                    self._partials_ptr, self._dev_ptr, stream), "co3_adamw_clipped")
        else:
            state = None
            if self._device_steps:
                state = self._dev_ptr
                B._chk(B._lib.co3_step_begin(self._args_ref, None, 0, self._lr_ptr, state, stream), "co3_step_begin")
            else:
                self._args.t = self._t + 1
            B._chk(self._step_fn(t.layout_ref, t.plan_ptr, self._master_ptr, *self._state_ptrs, self._args_ref, state, stream), "co3_adamw")
            if state is None:
                self._t += 1
        torch.autograd.graph.increment_version(t.params)       # written in place, though not by torch


class MixedAdamW:
    """AdamW over parameters of several types, as of a 16-bit model with 32-bit norms: one part (``AdamW``) per pair of parameter and
    gradient type, all of them one step, clipped by one norm.  Arguments as of ``AdamW``; ``master`` is for the 16-bit parts.
    ``parts`` hold the states, ``places[k]`` says which of the parameters part k has; the device counts the steps.  8-bit states are
    rounded by the seed, the step and the place within the part: equal places of two parts take equal random bits."""

    def __init__(self, params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], lr: Union[float, torch.Tensor] = 1e-3,
                 weight_decay: PerTensor = 0.01, lr_scales: PerTensor = 1.0, master: bool = False, max_norm: Optional[float] = None, **kw):
        params, grads = list(params), list(grads)
        if not params or len(params) != len(grads) or not all(isinstance(t, torch.Tensor) for t in params + grads):
            raise ValueError("gradients: one per parameter")
        if any(p.device != params[0].device for p in params):
            raise ValueError("parameters: all on one device")
        if max_norm is not None and not max_norm > 0.0:
            raise ValueError("max_norm must be positive")
        decays, scales = _per_tensor(weight_decay, len(params), "weight_decay"), _per_tensor(lr_scales, len(params), "lr_scales")
        kw.pop("device_steps", None)                                # always so
        if _overlapping(params, grads):
            raise ValueError("a parameter shares memory with another one or with a gradient")
        kinds = {}
        for k, (p, g) in enumerate(zip(params, grads)):
            kinds.setdefault((p.dtype, g.dtype), []).append(k)
        self.places = list(kinds.values())
        pick = lambda values, places: [values[k] for k in places]  # noqa: E731
        self.parts = [AdamW(pick(params, places), pick(grads, places), lr=lr, weight_decay=pick(decays, places),
                            lr_scales=pick(scales, places), master=master and ptype != torch.float32, device_steps=True, **kw)
                      for (ptype, _), places in kinds.items()]
        self.max_norm = max_norm
        first = self.parts[0]
        first._args.max_norm = math.inf if max_norm is None else max_norm
        self._dev, self.norm = first._dev, first.norm               # the one count, norm and factor of all parts
        counts = [part._table.layout.partials for part in self.parts]
        self._partials = torch.zeros(sum(counts), dtype=torch.float64, device=self._dev.device)
        at = [sum(counts[:k]) for k in range(len(counts))]
        self._partials_ptrs = [C.c_void_p(self._partials.data_ptr() + 8 * a) for a in at]
        for part in self.parts:
            part._table.also += [self._dev, self._partials]
        self._table = first._table
        torch.cuda.current_stream(self._dev.device).synchronize()      # cleared, for whichever stream comes first

    @property
    def lr(self):
        return self.parts[0].lr

    @lr.setter
    def lr(self, lr):
        for part in self.parts:
            part.lr = lr

    @property
    def t(self) -> int:
        """Number of steps taken (waits for the device)."""
        return self.parts[0].t

    @t.setter
    def t(self, t: int):
        self.parts[0].t = t

    @property
    def skipped(self) -> int:
        """Steps left out because their norm was not finite (waits for the device)."""
        return self.parts[0].skipped

    def take_masters(self):
        """Masters as the parameters are now (after the parameters were loaded from elsewhere)."""
        for part in self.parts:
            part.take_masters()

    def moments(self):
        """(m, v) of every tensor as float32 copies, in the parameters' order."""
        out = {}
        for places, part in zip(self.places, self.parts):
            out.update(zip(places, part.moments()))
        return [out[k] for k in sorted(out)]

    def state_dict(self) -> dict:
        return {"parts": [part.state_dict() for part in self.parts]}

    def load_state_dict(self, d: dict):
        """All of a state, or, where some of it is missing or does not fit, nothing (ValueError)."""
        if not isinstance(d.get("parts"), (list, tuple)) or len(d["parts"]) != len(self.parts):
            raise ValueError("state_dict: of another number of parts")
        for part, s in zip(self.parts, d["parts"]):
            part._check_state(s)
        for part, s in zip(self.parts, d["parts"]):
            part.load_state_dict(s)

    @_on_device
    def step(self, grads: Optional[Sequence[torch.Tensor]] = None):
        """One step on every tensor.  ``grads``: None, or tensors of the same sizes and types to take instead, from now on."""
        if grads is not None and len(grads) != sum(len(places) for places in self.places):
            raise ValueError("gradients: one per parameter")
        for part in self.parts:
            part._look_at_lr()
        tables = [part._table for part in self.parts]
        was = [t.now() for t in tables]
        try:
            for places, t in zip(self.places, tables):
                stream = t.ready(None if grads is None else [grads[k] for k in places])
            # a part's plan is checked against its own tensors: one that is new, against the other parts' too
            if any(t.plan is not w[1] for t, w in zip(tables, was)) and _overlapping([p for t in tables for p in t.params],
                                                                                     [g for t in tables for g in t.grads]):
                raise ValueError("a parameter shares memory with another one or with a gradient")
        except Exception:
            for t, w in zip(tables, was):                           # what was refused is not kept, by any part
                t.back(w)
            raise
        first, partials = self.parts[0], None
        if self.max_norm is not None:
            partials = self._partials_ptrs[0]
            for part, at in zip(self.parts, self._partials_ptrs):
                t = part._table
                B._chk(B._lib.co3_grad_sumsq(t.layout_ref, t.plan_ptr, at, stream), "co3_grad_sumsq")
        B._chk(B._lib.co3_step_begin(first._args_ref, partials, self._partials.numel(), first._lr_ptr, first._dev_ptr, stream),
               "co3_step_begin")
        for part in self.parts:
            t = part._table
            B._chk(part._step_fn(t.layout_ref, t.plan_ptr, part._master_ptr, *part._state_ptrs, part._args_ref, first._dev_ptr, stream),
                   "co3_adamw")
            torch.autograd.graph.increment_version(t.params)
