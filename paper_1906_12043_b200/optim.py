"""Thin binding over AdamW of libcocod.so (include/cocod_adamw.h).

Marshalling only: moments, updates and their coding are computed by the library's CUDA kernels.  torch is used for device memory and
streams.  No CPU fallback.

    opt = AdamW(params, lr=3e-4, weight_decay=0.1, state_bits=8)     # any number of tensors, one launch
    opt.step(grads)                                                  # or opt.step(): the parameters' .grad

    opt = EngineAdamW(engine, [(n, decay), ...], lr=3e-4)            # the K workers of an Engine
    opt.local_step(grads)                                            # in place of engine.local_step(grads)
"""
from __future__ import annotations

import contextlib
import ctypes
import math

import torch

from . import engine as _E

BLOCK = 128                      # values that share a unit in the 8-bit state; every tensor's moments start at a multiple of it


class _Moments:
    """What AdamW and EngineAdamW share: the moments, the clock and the handle."""

    def __init__(self, sizes, lr, betas, eps, weight_decay, state_bits, starts=None):
        if not torch.cuda.is_available():
            raise RuntimeError("AdamW needs a CUDA device (there is no CPU fallback)")
        if state_bits not in (8, 32):
            raise ValueError(f"state_bits: 8 or 32, got {state_bits}")
        n = len(sizes)
        decays = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
        if len(decays) != n:
            raise ValueError(f"weight_decay: one number, or one for each of the {n} tensors")
        self._lib = _E.load()
        from . import _lm_binding
        self._b = _lm_binding
        c_sizes = (ctypes.c_int64 * n)(*sizes)
        self.values = int(self._lib.cocod_adamw_values(n, c_sizes))
        if self.values < 0:
            raise ValueError("need at least one tensor, and none without values")
        self._device = torch.cuda.current_device()
        self.state_bits, self._lr = state_bits, float(lr)
        self.betas, self.eps = (float(betas[0]), float(betas[1])), float(eps)
        kinds = (torch.float32, torch.float32) if state_bits == 32 else (torch.int8, torch.uint8, torch.float32, torch.float32)
        self._state = [torch.zeros(self.values if i < 2 else self.values // BLOCK, dtype=k, device="cuda") for i, k in enumerate(kinds)]
        at = [t.data_ptr() for t in self._state] + [None, None]
        h = ctypes.c_void_p()
        rc = self._lib.cocod_adamw_create(ctypes.byref(h), n, c_sizes, (ctypes.c_float * n)(*decays), None if starts is None else (ctypes.c_int64 * n)(*starts),
                                          state_bits, *at[:4], self._lr, *self.betas, self.eps)
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_adamw_create")
        self._h = h.value
        with self._in_order():                  # (the first step may come on another stream than the zeros)
            pass

    def _ck(self, rc, name):
        if rc != _E.OK:
            raise _E.CocodError(rc, name)

    def _own_stream(self):
        """None: everything is ordered on torch's current stream."""
        return None

    def _stream(self):
        """The stream of the next call.  The handle's device has to be the current one."""
        if not self._h:
            raise ValueError("the optimizer was destroyed")
        if torch.cuda.current_device() != self._device:
            raise ValueError(f"the current device is cuda:{torch.cuda.current_device()}, this optimizer was made on cuda:{self._device}: "
                             f"call it under torch.cuda.device({self._device})")
        own = self._own_stream()
        return torch.cuda.current_stream().cuda_stream if own is None else own

    @contextlib.contextmanager
    def _in_order(self):
        """The stream of the handle's calls (None: torch's current one).  Another than the current one works behind what that one holds, and the current one goes on
        behind what is done inside: so the current stream's tensors are read and written there, and used, changed or freed afterwards, in the order of the calls."""
        own = self._own_stream()
        if own is None:
            yield None
            return
        here, there = torch.cuda.current_stream(), torch.cuda.ExternalStream(own) if own else torch.cuda.default_stream()
        if here.cuda_stream == own:
            yield here
            return
        there.wait_stream(here)
        try:
            yield there
        finally:
            here.wait_stream(there)

    @property
    def lr(self) -> float:
        """The learning rate.  Setting it is ordered on the stream of the steps (EngineAdamW: the engine's compute stream); captured steps follow it."""
        return self._lr

    @lr.setter
    def lr(self, value: float):
        self._ck(self._lib.cocod_adamw_set_lr(self._h, float(value), self._stream()), "cocod_adamw_set_lr")
        self._lr = float(value)

    @property
    def steps(self) -> int:
        """Steps done (synchronises the stream of the steps)."""
        got = ctypes.c_int64()
        self._ck(self._lib.cocod_adamw_get_step(self._h, ctypes.byref(got), self._stream()), "cocod_adamw_get_step")
        return int(got.value)

    def _flat(self, t, name):
        if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or not t.is_cuda or t.get_device() != self._device or not t.is_contiguous() \
                or t.numel() != self.values or t.data_ptr() % 16:
            raise ValueError(f"{name}: need {self.values} contiguous float32 values on cuda:{self._device}, 16-byte aligned")
        return t.data_ptr()

    def moments(self):
        """(m, v) in float32, the tensors one behind the other, each starting at a multiple of 128 values.  A copy; of an AdamW with 32 bits the state itself, which its
        next step changes.  (An engine's is a copy always: its steps run on another stream than what reads the moments.)"""
        if self.state_bits == 32 and self._own_stream() is None:
            return tuple(self._state)
        with self._in_order():
            both = self._b.adamw_moments(self._h, self._device, self.values, self._state[0], self._own_stream())
        if type(both) is int:
            raise _E.CocodError(both, "cocod_adamw_moments")
        return both

    def load_moments(self, steps: int, m, v):
        """Continue after `steps` steps with these moments (float32, as moments() returns them; what lies between the tensors has to be 0)."""
        stream, at = self._stream(), (self._flat(m, "m"), self._flat(v, "v"))
        if steps < 0:
            raise ValueError(f"steps: 0 or more, got {steps}")
        with self._in_order():
            self._ck(self._lib.cocod_adamw_load(self._h, *at, stream), "cocod_adamw_load")
        self._ck(self._lib.cocod_adamw_set_step(self._h, int(steps), stream), "cocod_adamw_set_step")

    def state_dict(self):
        """A copy of the state as it is held."""
        steps, copies = self.steps, [torch.empty_like(t) for t in self._state]
        with self._in_order() as there, torch.cuda.stream(there):
            for a, b in zip(copies, self._state):
                a.copy_(b)
        return {"state_bits": self.state_bits, "steps": steps, "lr": self.lr, "state": copies}

    def load_state_dict(self, d):
        stream = self._stream()
        if d["state_bits"] != self.state_bits or len(d["state"]) != len(self._state) or \
                any(a.shape != b.shape or a.dtype != b.dtype for a, b in zip(d["state"], self._state)):
            raise ValueError("the state of another model, or with another number of bits")
        steps, lr = int(d["steps"]), float(d["lr"])
        if steps < 0 or not math.isfinite(lr):
            raise ValueError(f"a state after {steps} steps with the rate {lr}")
        with self._in_order() as there, torch.cuda.stream(there):
            for a, b in zip(self._state, d["state"]):
                a.copy_(b)
        self._ck(self._lib.cocod_adamw_set_step(self._h, steps, stream), "cocod_adamw_set_step")
        self.lr = lr

    def __reduce__(self):
        raise TypeError("an optimizer is not copied or pickled: save its state_dict(), and load it into another one")

    @property
    def launch_count(self) -> int:
        return int(self._lib.cocod_adamw_launch_count(self._h))

    def destroy(self):
        if getattr(self, "_h", 0):
            h, self._h = self._h, 0
            self._lib.cocod_adamw_destroy(h)

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class AdamW(_Moments):
    """AdamW over a list of contiguous CUDA tensors, all bf16 or all float32, that do not overlap."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay=0.01, state_bits: int = 32, copies=None):
        """weight_decay: one number, or one for each tensor.  state_bits: 32, or 8 (blocks of 128 values share a unit).  copies: bf16 tensors that are
        written with float32 parameters, for example those that products read (None in the list: that one has none)."""
        self.params = tuple(params)             # (as many and as large as the state: step refuses others)
        if not self.params or any(not isinstance(p, torch.Tensor) for p in self.params):
            raise ValueError("params: need tensors")
        self.copies = None if copies is None else tuple(copies)
        written = [t for t in self.params + (self.copies or ()) if t is not None]
        if len({t.data_ptr() for t in written}) != len(written):
            raise ValueError("params: a tensor is there twice")
        if self.copies is not None and (len(self.copies) != len(self.params) or self.params[0].dtype != torch.float32):
            raise ValueError("copies: one for each float32 parameter (None: none)")
        super().__init__([p.numel() for p in self.params], lr, betas, eps, weight_decay, state_bits)

    def step(self, grads=None, grad_scale=None):
        """One step on torch's current stream (order the steps of one object).  grads: one for each parameter, all bf16 or all float32 (default: the parameters' .grad); a parameter whose
        gradient is None keeps its value and its moments (the number of steps, by which moments are corrected, is the optimizer's).  grad_scale: one float32 on the device, a factor of all gradients."""
        if grads is None:
            grads = [p.grad for p in self.params]
        rc = self._b.adamw_step(self._h, self._device, self.params, grads if type(grads) in (list, tuple) else list(grads), self.copies, grad_scale)
        if rc != _E.OK:
            raise _E.CocodError(rc, "cocod_adamw_step")


class EngineAdamW(_Moments):
    """AdamW as the local step of an Engine's K workers (moments for each of them)."""

    def __init__(self, engine, tensors=None, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, state_bits: int = 32):
        """tensors: [(values, weight decay), ...] of one worker's model, one behind the other; what is left of its P values is one more tensor without decay."""
        tensors = [(int(n), float(d)) for n, d in (tensors or [])]
        left = engine.P - sum(n for n, _ in tensors)
        if left < 0 or any(n < 1 for n, _ in tensors):
            raise ValueError(f"tensors: they have to fit the model's {engine.P} values, each at least one")
        if left:
            tensors.append((left, 0.0))
        sizes, decays, starts = [], [], []
        for i in range(engine.K):
            at = i * engine.P
            for n, d in tensors:
                sizes.append(n), decays.append(d), starts.append(at)
                at += n
        self.engine = engine
        super().__init__(sizes, lr, betas, eps, decays, state_bits, starts)

    def _own_stream(self):
        """The engine's compute stream: everything here is ordered there, as the engine's own calls are, and what goes in and out with the current stream."""
        return self.engine._compute

    def local_step(self, grads, grad_scale=None):
        """Step II, one iteration for all workers, on the engine's compute stream.  grads: K x P float32 CUDA tensor, complete and kept in that stream's order, as
        Engine.local_step's."""
        self._stream()
        e = self.engine
        if not e._h:
            raise ValueError("the engine was destroyed")
        if e._check_tensor(grads, e.K * e.P, "grads") != 0:
            raise ValueError("grads must be a CUDA tensor")
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or not grad_scale.is_cuda or grad_scale.numel() != 1):
            raise ValueError("grad_scale: need one float32 on the device")
        for t, name in ((grads, "grads"), (grad_scale, "grad_scale")):
            if t is not None and t.get_device() != self._device:
                raise ValueError(f"{name}: on cuda:{t.get_device()}, need cuda:{self._device} (the current device at creation)")
        self._ck(self._lib.cocod_adamw_local_step(self._h, e._h, _E._ptr(grads), _E._ptr(grad_scale)), "cocod_adamw_local_step")
