"""AdamW over many tensors, and the norm of their gradients: holders of the contexts of include/qadam.h.

Both run on the current stream of their device, so they can be captured into a CUDA graph as torch's own
operations are.  Gradients are bound once (a training program keeps its gradient buffers) and again when
they move.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple, Union

import torch

from .binding import AdamWBuffers, AdamWConfig, BF16, F16, F32, TensorList, _check, load_library

TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}


def element_type(dtype: torch.dtype, what: str) -> int:
    if dtype not in TYPES:
        raise ValueError(f"{what}: {dtype} is not offered (float32, bfloat16 or float16)")
    return TYPES[dtype]


def stream_of(device: torch.device) -> int:
    """The device's current stream (torch.cuda.current_stream(device).cuda_stream, without the object: 0.1 us, not 2)."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _device_of(tensors: Sequence[Optional[torch.Tensor]], what: str) -> torch.device:
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or next(iter(devices)).type != "cuda":
        raise ValueError(f"{what} must be CUDA tensors of one device; there is no CPU path")
    return next(iter(devices))


def _need_cuda() -> None:
    load_library()
    if not torch.cuda.is_available():
        raise RuntimeError("paper_2004_14180_b200 needs a CUDA device; there is no CPU path")


def _pointers(tensors: Sequence[Optional[torch.Tensor]]):
    return (C.c_void_p * len(tensors))(*[t.data_ptr() if t is not None and t.numel() else None for t in tensors])


def written(t: torch.Tensor) -> None:
    """Tells autograd that a call writes `t` by its address: a backward pass that needs what was there before is then refused,
    as it is after torch's own in-place operations.  (torch.autograd.graph.increment_version without its look at the
    argument: 0.2 us, not 0.35.)"""
    if not t.is_inference():
        torch._C._increment_version((t,))


def _check_bound(tensors, lens, types, device, what: str) -> None:
    if len(tensors) != len(lens):
        raise ValueError(f"{len(tensors)} {what} for {len(lens)} tensors")
    for i, (t, n, ty) in enumerate(zip(tensors, lens, types)):
        if t is None:
            continue
        if t.device != device or t.numel() != n or t.dtype not in TYPES or TYPES[t.dtype] != ty or not t.is_contiguous():
            raise ValueError(f"{what}[{i}]: a contiguous tensor of {n} elements on {device}, of the type that the context was "
                             f"created for, is needed; got {tuple(t.shape)} {t.dtype} on {t.device}")


class _Scratch:
    def __init__(self, size: int, device: torch.device):
        self.buf = torch.empty(size + 256, dtype=torch.uint8, device=device)
        self.ptr = (self.buf.data_ptr() + 255) // 256 * 256
        self.size = size


class GradNorm:
    """sqrt of the sum of squares over all tensors, and the factor that clips it.

    tensors: contiguous CUDA tensors of float32, bfloat16 or float16, of any lengths.  Calls of one holder
    share scratch: order them (one stream, or events).  Keep the holder until its calls are done, and as long as a graph that
    captured one is replayed.
    """

    ctx = None

    def __init__(self, tensors: Sequence[torch.Tensor]):
        _need_cuda()
        tensors = list(tensors)
        if not tensors:
            raise ValueError("no tensors")
        self._create([t.numel() for t in tensors], [element_type(t.dtype, "tensors") for t in tensors], _device_of(tensors, "tensors"))
        self.bind(tensors)

    @classmethod
    def _of(cls, lens: Sequence[int], types: Sequence[int], device: torch.device) -> "GradNorm":
        """One for tensors of these lengths and types, none of them bound."""
        norm = cls.__new__(cls)
        norm._create(lens, types, device)
        return norm

    def _create(self, lens: Sequence[int], types: Sequence[int], device: torch.device) -> None:
        self.device, self._lens, self._types = device, list(lens), list(types)
        n = len(self._lens)
        spec = TensorList(n, 0, (C.c_int64 * n)(*self._lens), (C.c_int32 * n)(*self._types))
        size, ctx = C.c_size_t(), C.c_void_p()
        L = load_library()
        _check(L.qadam_norm_query_sizes(C.byref(spec), C.byref(size)), "qadam_norm_query_sizes")
        with torch.cuda.device(self.device):
            self._scratch = _Scratch(size.value, self.device)
            torch.cuda.current_stream(self.device).synchronize()      # its memory may still be in use there
            _check(L.qadam_norm_create(C.byref(spec), self._scratch.ptr, size.value, C.byref(ctx)), "qadam_norm_create")
        self.ctx = ctx.value
        # (not filled: a fill here would run on this stream, after a first call on another)
        self.result = torch.empty(2, dtype=torch.float32, device=self.device)

    def bind(self, tensors: Sequence[Optional[torch.Tensor]]) -> None:
        """The tensors that later calls read, of the lengths and types given at creation; None counts as zero."""
        tensors = list(tensors)
        _check_bound(tensors, self._lens, self._types, self.device, "tensors")
        _check(load_library().qadam_norm_bind(self.ctx, _pointers(tensors)), "qadam_norm_bind")
        self._bound = tensors

    def __call__(self, max_norm: float = float("inf"), out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """-> (norm, factor), float32 scalars on the device; views of `out` ([2] float32), or of a buffer that the next
        call overwrites.  The factor is NaN where the norm is not finite."""
        out = self.result if out is None else out
        if out.device != self.device or out.dtype != torch.float32 or out.numel() != 2 or not out.is_contiguous():
            raise ValueError("out: two contiguous float32 on the tensors' device are needed")
        _check(load_library().qadam_norm_run(self.ctx, max_norm, out.data_ptr(), stream_of(self.device)), "qadam_norm_run")
        written(out)
        return out[0], out[1]

    @property
    def launches(self) -> int:
        return int(load_library().qadam_norm_launch_count(self.ctx))

    def close(self) -> None:
        if self.ctx:
            load_library().qadam_norm_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW:
    """AdamW over a list of tensors (formulas, layout and 8-bit moments: include/qadam.h).

    weights, grads: contiguous CUDA tensors of float32, bfloat16 or float16, in any mix.  A grad may be
    None: it then has its weight's type, and its tensor is left as it is until `bind` brings one.
    state_bits: 32, or 8 (moments in one byte each and two scales per 128 elements, rounded at random by `seed`).
    master: keep float32 master weights (`self.master`, padded layout; set from `weights` here).
    weight_decay: one factor, or one for each tensor.
    Moments are `m`, `v` ([D] float32, padded layout) or `m`, `r` ([D] uint8) with `m_scale`, `r_scale`.
    Weights are updated in place, where they are now, and autograd is told so (but for replays of a captured step).  Steps run on the
    current stream; keep the holder until they are done, and as long as a graph that captured them is replayed (with the gradients
    that were bound at its capture).
    Creating one writes its tables to the device and waits (2 ms for 109.5 x 10^6 elements in 199 tensors; the first grad_norm 0.5).
    """

    ctx = None

    def __init__(self, weights: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]], state_bits: int = 32,
                 master: bool = False, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, lr: float = 1e-3,
                 weight_decay: Union[float, Sequence[float]] = 0.0, seed: int = 0):
        _need_cuda()
        weights, grads = list(weights), list(grads)
        self.weights = [w.detach() for w in weights]
        if not self.weights or len(grads) != len(self.weights):
            raise ValueError(f"{len(grads)} gradients for {len(self.weights)} weights")
        self.device = _device_of(self.weights, "weights")
        n = len(self.weights)
        self._lens = [w.numel() for w in self.weights]
        wtypes = [element_type(w.dtype, "weights") for w in self.weights]
        if not all(w.is_contiguous() for w in self.weights):
            raise ValueError("weights must be contiguous")
        self._types = [element_type((g if g is not None else w).dtype, "grads") for g, w in zip(grads, self.weights)]
        end = 0
        for first, size in sorted((w.data_ptr(), w.numel() * w.element_size()) for w in self.weights if w.numel()):
            if first < end:
                raise ValueError("weights overlap: a tensor may be listed once only")
            end = first + size
        decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
        if len(decay) != n:
            raise ValueError(f"{len(decay)} weight decays for {n} weights")
        self.state_bits = state_bits
        cfg = AdamWConfig(n, state_bits, (C.c_int64 * n)(*self._lens), (C.c_int32 * n)(*wtypes), (C.c_int32 * n)(*self._types),
                          (C.c_float * n)(*decay), beta1, beta2, eps, lr, int(master), 0, seed & 0xFFFFFFFFFFFFFFFF)
        L = load_library()
        D, off, size = C.c_int64(), (C.c_int64 * n)(), C.c_size_t()
        _check(L.qadam_adamw_query_sizes(C.byref(cfg), C.byref(D), off, C.byref(size)), "qadam_adamw_query_sizes")
        self.D, self.off = D.value, list(off)
        room = max(self.D, 4)                        # a set of empty tensors still has addresses
        with torch.cuda.device(self.device):
            z = lambda k, dtype=torch.float32: torch.zeros(k, dtype=dtype, device=self.device)  # noqa: E731
            eight = state_bits == 8
            self.m = z(room, torch.uint8 if eight else torch.float32)[:self.D]
            second = z(room, torch.uint8 if eight else torch.float32)[:self.D]
            self.v, self.r = (None, second) if eight else (second, None)
            self.m_scale, self.r_scale = (z(room // 128 + 4)[:self.D // 128], z(room // 128 + 4)[:self.D // 128]) if eight else (None, None)
            self.master = z(room)[:self.D] if master else None
            if master:
                torch._foreach_copy_([self.master[o:o + k] for o, k in zip(self.off, self._lens)], [w.view(-1) for w in self.weights])
            self.count = torch.zeros(1, dtype=torch.int64, device=self.device)
            self.status = torch.zeros(1, dtype=torch.int32, device=self.device)
            self._scratch = _Scratch(size.value, self.device)
            at = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
            bufs = AdamWBuffers(_pointers(self.weights), at(self.master), at(self.m), at(second), at(self.m_scale), at(self.r_scale),
                                self.count.data_ptr(), self._scratch.ptr, size.value, self.status.data_ptr())
            torch.cuda.current_stream(self.device).synchronize()
            ctx = C.c_void_p()
            _check(L.qadam_adamw_create(C.byref(cfg), C.byref(bufs), C.byref(ctx)), "qadam_adamw_create")
        self.ctx = ctx.value
        # what counts the writes to the weights: one for all views of a tensor
        self._counted = list({id(w if w._base is None else w._base): w for w in weights if not w.is_inference()}.values())
        self._norm: Optional[GradNorm] = None
        self.bind(grads)

    def bind(self, grads: Sequence[Optional[torch.Tensor]]) -> None:
        """The gradients that later steps read, of the lengths and types given at creation; None leaves a tensor as it is."""
        grads = list(grads)
        _check_bound(grads, self._lens, self._types, self.device, "grads")
        _check(load_library().qadam_adamw_bind(self.ctx, _pointers(grads)), "qadam_adamw_bind")
        self.grads = grads
        if self._norm is not None:
            self._norm.bind(grads)

    def grad_norm(self, max_norm: float = float("inf")) -> Tuple[torch.Tensor, torch.Tensor]:
        """(norm of all bound gradients, factor that clips it to max_norm): see GradNorm.  The first call makes its context,
        so make it outside any stream capture."""
        if self._norm is None:
            norm = GradNorm._of(self._lens, self._types, self.device)
            norm.bind(self.grads)
            self._norm = norm
        return self._norm(max_norm)

    def _scalar(self, t: torch.Tensor, what: str) -> int:
        if t.device != self.device or t.dtype != torch.float32 or t.numel() != 1:
            raise ValueError(f"{what}: one float32 on {self.device} is needed")
        return t.data_ptr()

    def step(self, step: int, lr: Optional[float] = None, grad_scale: Optional[torch.Tensor] = None) -> None:
        """Step number `step` (from 1).  grad_scale: one float32 on the device that every gradient is multiplied by; if it is
        not finite the step changes nothing and sets ST_NONFINITE.  A captured call repeats its number and lr."""
        if lr is not None and not lr >= 0:
            raise ValueError("lr must be >= 0")
        rc = load_library().qadam_adamw_step(self.ctx, step, -1.0 if lr is None else lr,
                                             None if grad_scale is None else self._scalar(grad_scale, "grad_scale"),
                                             stream_of(self.device))
        if rc:
            _check(rc, "qadam_adamw_step")
        torch._C._increment_version(self._counted)

    def step_counted(self, lr: Optional[torch.Tensor] = None, grad_scale: Optional[torch.Tensor] = None) -> None:
        """The step after the `count` (int64 on the device) that have been taken, with lr read from the device: for a step that
        is captured once and replayed."""
        rc = load_library().qadam_adamw_step_counted(self.ctx, None if lr is None else self._scalar(lr, "lr"),
                                                     None if grad_scale is None else self._scalar(grad_scale, "grad_scale"),
                                                     stream_of(self.device))
        if rc:
            _check(rc, "qadam_adamw_step_counted")
        torch._C._increment_version(self._counted)

    def moments(self, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(m, v) as float32, padded layout: the buffers themselves, or 8-bit moments decoded (into `out` if given)."""
        if self.state_bits == 32:
            if out is not None:
                raise ValueError("32-bit moments are the buffers themselves: there is nothing to decode")
            return self.m, self.v
        if out is None:
            out = (torch.empty(self.D, dtype=torch.float32, device=self.device), torch.empty(self.D, dtype=torch.float32, device=self.device))
        for t in out:
            if t.device != self.device or t.dtype != torch.float32 or t.numel() != self.D or not t.is_contiguous():
                raise ValueError(f"out: two contiguous float32 tensors of {self.D} elements are needed")
        if self.D:
            _check(load_library().qadam_adamw_moments(self.ctx, out[0].data_ptr(), out[1].data_ptr(), stream_of(self.device)),
                   "qadam_adamw_moments")
            for t in out:
                written(t)
        return out

    def view(self, buffer: torch.Tensor, i: int) -> torch.Tensor:
        """Tensor i's part of a padded buffer ([D]: master, m, v), in the shape of its weight."""
        return buffer[self.off[i]:self.off[i] + self._lens[i]].view(self.weights[i].shape)

    def poll_status(self) -> int:
        """Waits for the current stream; bits of the status word (ST_NONFINITE)."""
        st = C.c_uint32()
        _check(load_library().qadam_adamw_poll_status(self.ctx, stream_of(self.device), C.byref(st)), "qadam_adamw_poll_status")
        return st.value

    @property
    def launches(self) -> int:
        return int(load_library().qadam_adamw_launch_count(self.ctx))

    def close(self) -> None:
        if self.ctx:
            load_library().qadam_adamw_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
