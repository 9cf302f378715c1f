"""AdamW over many tensors in one call, with states in 32 or in 8 bits, on this library's kernel.

    optimizer = AdamW(params, lr=1e-3, state_bits=8)          # fp32 or bf16 CUDA tensors, one dtype
    optimizer = AdamW(masters, copies=weights)                # fp32 masters and the bf16 tensors the layers multiply with
    optimizer.step(grads)                                     # or step(): the params' .grad

An 8-bit state holds e4m3 codes (``torch.float8_e4m3fn`` tensors of the parameters' shapes) with one power of two for each
256 elements, the first moment and the square root of the second, rounded up or down at random by the library's counter
hash of ``seed + step``: a step can be repeated bit for bit.  16 bytes of memory traffic an element instead of 28 with an
fp32 parameter and gradient.
"""
from __future__ import annotations

import ctypes
from operator import attrgetter

import torch
from torch.autograd.graph import increment_version

from . import binding

BLOCK = 256   # elements that share a scale


def _array(addresses):
    return (ctypes.c_void_p * len(addresses))(*addresses)


_dtype_of, _shape_of = attrgetter("dtype"), attrgetter("shape")


# One call that looks at dtype, device, shape and strides of a list of tensors, where this torch has it.  It stands in for a check in
# Python that found the same list in order (161 tensors: 16 us instead of 56); what it does not recognise is checked again.
_guards = getattr(getattr(torch._C, "_dynamo", None), "guards", None)


def _recognise(tensors):
    """A function of tensors: whether they are, in all that ``_check`` looks at and in shape, what these here are."""
    guard = getattr(_guards, "TensorGuards", None)
    if guard is None:
        return lambda *_: False
    return guard(*tensors, dynamic_dims_sizes=[list(t.shape) for t in tensors], dynamic_dims_strides=[list(t.stride()) for t in tensors]).check


def _layout(p: torch.Tensor):
    """The order of a param's elements in memory, which has no gaps: the one of its axes, or channels last."""
    for layout in (torch.contiguous_format, torch.channels_last):
        if (layout is torch.contiguous_format or p.dim() == 4) and p.is_contiguous(memory_format=layout):
            return layout
    raise ValueError("params must be contiguous, or four-dimensional with the channels last")


def _in_order(tensors, layouts) -> bool:
    """Whether the tensors lie as the params do (``layouts``: theirs, None where all are contiguous)."""
    if layouts is None:
        return all(map(torch.Tensor.is_contiguous, tensors))
    return len(tensors) == len(layouts) and all(t.is_contiguous(memory_format=k) for t, k in zip(tensors, layouts) if t.dim() == 4 or k is torch.contiguous_format)


def _check(tensors, name: str, dtype=None, layouts=None):
    """One dtype (this one, where it is given), one GPU, laid out as the params; returns the dtype."""
    if not _in_order(tensors, layouts):
        raise ValueError(f"{name} must be contiguous, or lie in memory as the params do")
    devices, dtypes = set(map(torch.Tensor.get_device, tensors)), set(map(_dtype_of, tensors))
    if tensors and min(devices) < 0:
        raise ValueError(f"{name} must live on the GPU")
    if len(dtypes | ({dtype} if dtype else set())) > 1 or len(devices) > 1:
        raise ValueError(f"{name} must have one dtype{f' ({dtype})' if dtype else ''} and one device")
    return next(iter(dtypes), torch.float32)


class AdamW:
    """Holds the states of ``params`` and steps them in place.

    Params are contiguous, or four-dimensional with the channels last; gradients, copies and states lie in memory as their
    param does, and an 8-bit state's blocks are runs of that memory.  Every param has a gradient in every step.
    ``copies``: bf16 tensors of the (fp32) params' shapes that every step writes the new values to as well.  ``state``:
    tensors to go on from instead of zeros, a dict of lists as ``state()`` returns it, ``steps`` the steps they have seen.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, *,
                 state_bits: int = 32, copies=None, seed: int = 0, state: dict | None = None, steps: int = 0):
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32")
        self.params = list(params)
        self.copies = None if copies is None else list(copies)
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.state_bits, self.seed, self.steps = state_bits, int(seed), int(steps)
        layouts = list(map(_layout, self.params))
        self._layouts = layouts if torch.channels_last in layouts else None
        self._dtype = _check(self.params, "params", None, self._layouts)
        self._device = self.params[0].get_device() if self.params else 0
        self._param_dt = binding._dtype_code(self.params[0]) if self.params else binding.F32
        self._numel, self._shapes = [p.numel() for p in self.params], [p.shape for p in self.params]
        self._counts = (ctypes.c_int64 * len(self.params))(*self._numel)
        if self.copies is not None and self._dtype != torch.float32:
            raise ValueError("copies are for fp32 params")
        if state is None:
            state = self._zeros()
        names = ("exp_avg", "exp_avg_sq") + (("exp_avg_scale", "exp_avg_sq_scale") if state_bits == 8 else ())
        if set(state) != set(names):
            raise ValueError(f"state holds {', '.join(names)}")
        self._state = {k: [t.detach() for t in state[k]] for k in names}
        # the states of one storage move together: one of them tells of all
        self._followed = list({t.untyped_storage().data_ptr(): t for ts in self._state.values() for t in ts if t.numel()}.values())
        self._seen, self._arrays, self._same, self._same_grads = None, None, lambda *_: False, lambda *_: False
        self._places()
        # what autograd has to know of: a graph that saved one of these must not go back through the new values
        self._written = [t for t in (*self.params, *(self.copies or ())) if not t.is_inference()]

    def _places(self):
        """(params, copies, states): arrays of addresses, None for what there is not.

        Where the tensors are is looked at in every step: the caller may give params and copies new storage, and free and allocate
        the states', which whoever holds state() shares.  Params and copies are the caller's objects, so their strides, shapes and
        dtypes may change too, without a new address, and are looked at as well; the states' are aliases of the optimizer's own."""
        theirs = self.params if self.copies is None else self.params + self.copies
        now = list(map(torch.Tensor.data_ptr, theirs + self._followed))
        if now != self._seen or not self._same(*theirs):
            self._check_list("params", self.params)
            if self.copies is not None:
                self._check_list("copies", self.copies)
            for name, tensors in self._state.items():
                self._check_list(name, tensors)
            self._check_places()
            lists = (self.params, self.copies, *self._state.values())
            self._arrays = [None if ts is None else _array([t.data_ptr() for t in ts]) for ts in lists]
            self._seen, self._same = now, _recognise(theirs)
        params, copies, *states = self._arrays
        return params, copies, states

    def _check_list(self, name: str, tensors) -> None:
        """What the tensors are: all that the kernel takes for granted of them but where they are."""
        scales = name.endswith("_scale")
        _check(tensors, name, {"params": self._dtype, "copies": torch.bfloat16}.get(name) or
               (torch.float32 if scales or self.state_bits == 32 else torch.float8_e4m3fn), None if scales else self._layouts)
        if scales and [t.numel() for t in tensors] != [-(-n // BLOCK) for n in self._numel]:
            raise ValueError(f"{name} holds one value for each {BLOCK} elements of every param")
        if not scales and list(map(_shape_of, tensors)) != self._shapes:
            raise ValueError(f"{name} must have the shapes of params")
        if tensors and tensors[0].get_device() != self._device:
            raise ValueError(f"{name} must live on the GPU that the optimizer was made on")

    def _check_grads(self, grads) -> None:
        if any(g is None for g in grads):
            raise ValueError("one gradient for each param")
        dtypes = {g.dtype for g in grads}
        if len(dtypes) != 1 or not _in_order(grads, self._layouts) or [g.shape for g in grads] != self._shapes:
            raise ValueError("gradients must lie in memory as the params do, be of one dtype and of the params' shapes")
        if set(map(torch.Tensor.get_device, grads)) != {self._device}:
            raise ValueError("gradients must live on the params' GPU")

    def _check_places(self) -> None:
        """All that a step writes lies apart and within its storage.  (Two workgroups would step an element at once.)"""
        spans = []
        for t in (t for ts in (self.params, self.copies or (), *self._state.values()) for t in ts):
            size = t.nbytes
            if size == 0:
                continue
            storage, begin = t.untyped_storage(), t.data_ptr()
            if begin + size > storage.data_ptr() + storage.nbytes():
                raise ValueError("the storage of a param, copy or state is not there")
            spans.append((begin, begin + size))
        spans.sort()
        if any(end > begin for (_, end), (begin, _) in zip(spans, spans[1:])):
            raise ValueError("a tensor is twice among params, copies and states, or two of them share memory")

    def _zeros(self):
        def zeros():
            if self.state_bits == 32:
                return [torch.zeros_like(p, dtype=torch.float32) for p in self.params]
            return [torch.zeros_like(p, dtype=torch.uint8).view(torch.float8_e4m3fn) for p in self.params]   # e4m3's 0 is 0

        state = {"exp_avg": zeros(), "exp_avg_sq": zeros()}
        if self.state_bits == 8:
            for k in ("exp_avg_scale", "exp_avg_sq_scale"):
                state[k] = [torch.ones(-(-n // BLOCK), dtype=torch.float32, device=p.device) for n, p in zip(self._numel, self.params)]
        return state

    def state(self) -> dict:
        """The state by name, a list of tensors each in the order of the params; they share the optimizer's memory."""
        return {k: [t.detach() for t in v] for k, v in self._state.items()}

    def step(self, grads=None, *, grad_scale: torch.Tensor | None = None) -> None:
        """One step from ``grads`` (one dtype, fp32 or bf16; default: every param's ``.grad``, which must be there).
        ``grad_scale``: an fp32 tensor of one element on the GPU that the gradients are multiplied with (clipping, loss
        scaling).  Not inside a captured graph, whose replays would all be this one step."""
        grads = [p.grad for p in self.params] if grads is None else list(grads)
        if len(grads) != len(self.params):
            raise ValueError("one gradient for each param")
        if not grads:
            self.steps += 1
            return
        if not self._same_grads(*grads):
            self._check_grads(grads)
            self._same_grads = _recognise(grads)
        if grad_scale is not None and (grad_scale.get_device() != self._device or grad_scale.dtype != torch.float32 or grad_scale.numel() != 1):
            raise ValueError("grad_scale must be one float32 on the params' GPU")
        step = self.steps + 1
        params, copies, states = self._places()
        m, v, m_scale, v_scale = states if self.state_bits == 8 else (*states, None, None)
        rc = binding.load().sdgp_adamw_step(
            len(grads), params, _array(list(map(torch.Tensor.data_ptr, grads))), m, v, m_scale, v_scale,
            copies, self._counts, self._param_dt, binding._dtype_code(grads[0]), self.state_bits, self.lr,
            *self.betas, self.eps, self.weight_decay, step, binding._ptr(grad_scale), (self.seed + step) & (2**64 - 1),
            binding._stream(grads[0]))
        if rc != 0:
            captured = torch.cuda.is_current_stream_capturing()
            raise binding.SdgpError(rc, "sdgp_adamw_step" + (" on a stream that is being captured" if captured else ""))
        increment_version(self._written)
        self.steps = step
