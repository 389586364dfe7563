"""Thin ctypes binding of the layer operators (C ABI in include/esrnn_layers.h): gated linear recurrence, group norm with
activation, AdamW over many tensors.

Argument marshalling only, as in binding.py: the classes own the buffers of a layer, every call runs in the library's
kernels on the current stream of the tensors' device (or the one given), and a failed call raises EsrnnError.  There is no fallback.
Tensors that a call names have to live until the stream has run it, as with any work of torch on that stream.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .binding import ESRNN_OK, EsrnnError, load_library

KINDS = {"smooth": 0, "decay": 1}
ACTIVATIONS = {"none": 0, "silu": 1}
ADAMW_BLOCK = 256


class RecurrenceShape(C.Structure):
    _fields_ = [("B", C.c_int32), ("T", C.c_int32), ("C", C.c_int32), ("kind", C.c_int32), ("dtype", C.c_int32)] + [
        (name, C.c_int64 * 2) for name in ("x_stride", "gate_stride", "out_stride", "grad_out_stride", "grad_x_stride",
                                           "grad_gate_stride")]


class GroupNormShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("N", "T", "C", "G", "activation", "dtype")] + [("eps", C.c_float)]


class AdamWTensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("copy", C.c_void_p), ("n", C.c_int64), ("weight_decay", C.c_float),
                ("grad_dtype", C.c_int32), ("copy_dtype", C.c_int32)]


class AdamWConfig(C.Structure):
    _fields_ = [(name, C.c_double) for name in ("lr", "beta1", "beta2", "eps", "clip_norm")] + [("seed", C.c_uint32)]


_lib = None


def _library():
    """The library with the signatures of include/esrnn_layers.h."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load_library()
    vp, i32, i64, size = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(C.c_size_t)
    rs = C.POINTER(RecurrenceShape)
    for name, args in {
        "esrnn_recurrence_workspace_bytes": [rs, size],
        "esrnn_recurrence_saved_bytes": [rs, size],
        "esrnn_recurrence_forward": [rs] + [vp] * 9,
        "esrnn_recurrence_backward": [rs] + [vp] * 11,
        "esrnn_recurrence_step": [i32] * 5 + [vp, i64, vp, i64, vp, vp, vp, i64, vp],
        "esrnn_group_norm_workspace_bytes": [C.POINTER(GroupNormShape), size],
        "esrnn_group_norm_forward": [C.POINTER(GroupNormShape)] + [vp] * 8,
        "esrnn_group_norm_backward": [C.POINTER(GroupNormShape)] + [vp] * 11,
        "esrnn_adamw_create": [C.POINTER(AdamWTensor), i32, i32, C.POINTER(vp)],
        "esrnn_adamw_destroy": [vp],
        "esrnn_adamw_state_elements": [vp, size],
        "esrnn_adamw_workspace_bytes": [vp, size],
        "esrnn_adamw_bind": [vp, vp, vp],
        "esrnn_adamw_update": [vp, C.POINTER(AdamWConfig), i32] + [vp] * 8,
    }.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, C.c_int
    _lib = lib
    return lib


_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _dtype(dtype) -> int:
    found = _DTYPES.get(dtype)
    if found is None:
        raise ValueError(f"elements are float32, bfloat16 or float16, got {dtype}")
    return found


def _choice(table, name, what):
    if name not in table:
        raise ValueError(f"{what} is one of {', '.join(table)}, got {name!r}")
    return table[name]


def _raise(status, what):
    if status != ESRNN_OK:
        raise EsrnnError(status, what)


# (torch.cuda.current_stream() builds an object around this number: 1.9 us of a call of 8)
_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _stream(stream, device) -> int:
    """The stream that a caller gives, which has to be one of `device` (else it is the device's current one).  The library launches on the current
    device: the callers below make `device` that first."""
    if stream.device != device:
        raise ValueError(f"the stream is one of {stream.device}, the tensors are on {device}")
    return stream.cuda_stream


def _bytes(fn, *args) -> int:
    n = C.c_size_t()
    _raise(fn(*args, C.byref(n)), fn.__name__)
    return int(n.value)


def _check(t, name, shape, dtype, device, dense=True):
    """The address of a tensor that has to be there."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} has to be {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if dense and not t.is_contiguous():
        raise ValueError(f"{name} has to be contiguous")
    return t.data_ptr()


def _check_optional(t, name, shape, dtype, device):
    return None if t is None else _check(t, name, shape, dtype, device)


def _cuda(device):
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"a GPU is needed, got {device}")
    return torch.device("cuda", torch.cuda.current_device()) if device.index is None else device


class GatedRecurrence:
    """h_t = a_t h_{t-1} + b_t over sequences of up to T positions, C channels each on its own, with gates from the caller:
    kind "smooth": a = 1 - sigmoid(gate), b = sigmoid(gate) x;  kind "decay": a = sigmoid(gate), b = x.

    Tensors are [B, T, C], with time_major [T, B, C]; x, gate, grad_out (and grad_x, grad_gate, where the caller gives them) may
    be strided in any way that keeps channels next to each other, as the two halves of one projection's result do.
    lengths: int32 [B], positions that exist; initial, grad_last: float32 [B, C] or None (zero).
    Owns out, last, the gradients and what the reverse pass needs, all overwritten by the next call; last may be that call's initial, and
    grad_initial the next reverse pass's grad_last (they are copied before)."""

    def __init__(self, B: int, T: int, C_: int, kind: str = "smooth", dtype=None, time_major: bool = False,
                 training: bool = True, device="cuda"):
        dtype = torch.float32 if dtype is None else dtype
        self.device, self.dtype, self.time_major, self.training = _cuda(device), dtype, time_major, training
        self._index = self.device.index
        self._lib = _library()
        s = RecurrenceShape()
        s.B, s.T, s.C, s.kind, s.dtype = int(B), int(T), int(C_), _choice(KINDS, kind, "kind"), _dtype(dtype)
        self._shape, self._ref = s, C.byref(s)
        workspace = _bytes(self._lib.esrnn_recurrence_workspace_bytes, self._ref)
        saved = _bytes(self._lib.esrnn_recurrence_saved_bytes, self._ref)
        self.workspace = torch.empty(workspace, dtype=torch.uint8, device=self.device)
        self._size = torch.Size((T, B, C_) if time_major else (B, T, C_))
        self._rows = torch.Size((B, C_))
        self.out = torch.empty(self._size, dtype=dtype, device=self.device)
        self.last = torch.empty(self._rows, dtype=torch.float32, device=self.device)
        self._out_ptr, self._last_ptr, self._workspace_ptr = self.out.data_ptr(), self.last.data_ptr(), self.workspace.data_ptr()
        self._elements(self.out, "out", s.out_stride)
        self._forward_done, self._saved_ptr, self._carried = False, None, None
        if training:
            self.saved = torch.empty(saved // 4, dtype=torch.float32, device=self.device)
            self.grad_x, self.grad_gate = (torch.empty(self._size, dtype=dtype, device=self.device) for _ in range(2))
            self.grad_initial = torch.empty(self._rows, dtype=torch.float32, device=self.device)
            self._saved_ptr, self._grad_initial_ptr = self.saved.data_ptr(), self.grad_initial.data_ptr()

    def _elements(self, t, name, field) -> int:
        at = _check(t, name, self._size, self.dtype, self.device, dense=False)
        outer, inner, channel = t.stride()
        if channel != 1 and self._size[2] != 1:
            raise ValueError(f"{name}: channels have to lie next to each other")
        field[0], field[1] = (inner, outer) if self.time_major else (outer, inner)
        return at

    def _lengths(self, lengths):
        return _check_optional(lengths, "lengths", self._rows[:1], torch.int32, self.device)

    def _states(self, t, name, own, stream):
        """The address of states that a call reads: of a copy, if they are the layer's `own` that the call overwrites."""
        if t is None:
            return None
        at = _check(t, name, self._rows, torch.float32, self.device)
        if at != own:
            return at
        if self._carried is None:
            self._carried = torch.empty_like(t)
        with torch.cuda.stream(stream):     # (None: the current one)
            self._carried.copy_(t)
        return self._carried.data_ptr()

    def forward(self, x, gate, lengths=None, initial=None, stream=None):
        """(out, last): all states in the element type, zero past the lengths, and the last one of every sequence in float32."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.forward(x, gate, lengths, initial, stream)
        s = self._shape
        x_ptr, gate_ptr = self._elements(x, "x", s.x_stride), self._elements(gate, "gate", s.gate_stride)
        _raise(self._lib.esrnn_recurrence_forward(
            self._ref, x_ptr, gate_ptr, self._lengths(lengths),
            self._states(initial, "initial", self._last_ptr, stream), self._out_ptr, self._last_ptr,
            self._saved_ptr, self._workspace_ptr,
            _raw_stream(self._index) if stream is None else _stream(stream, self.device)), "esrnn_recurrence_forward")
        self._forward_done = True
        return self.out, self.last

    def backward(self, x, gate, grad_out, lengths=None, grad_last=None, grad_x=None, grad_gate=None, stream=None):
        """(grad_x, grad_gate, grad_initial) for the forward pass last run, which had the same x, gate and lengths."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.backward(x, gate, grad_out, lengths, grad_last, grad_x, grad_gate, stream)
        if not self.training or not self._forward_done:
            raise EsrnnError(4, "GatedRecurrence.backward")
        grad_x = self.grad_x if grad_x is None else grad_x
        grad_gate = self.grad_gate if grad_gate is None else grad_gate
        s = self._shape
        x_ptr, gate_ptr = self._elements(x, "x", s.x_stride), self._elements(gate, "gate", s.gate_stride)
        d_ptr = self._elements(grad_out, "grad_out", s.grad_out_stride)
        gx_ptr = self._elements(grad_x, "grad_x", s.grad_x_stride)
        gg_ptr = self._elements(grad_gate, "grad_gate", s.grad_gate_stride)
        _raise(self._lib.esrnn_recurrence_backward(
            self._ref, x_ptr, gate_ptr, self._lengths(lengths), self._saved_ptr, d_ptr,
            self._states(grad_last, "grad_last", self._grad_initial_ptr, stream), gx_ptr, gg_ptr,
            self._grad_initial_ptr, self._workspace_ptr,
            _raw_stream(self._index) if stream is None else _stream(stream, self.device)), "esrnn_recurrence_backward")
        return grad_x, grad_gate, self.grad_initial


def recurrence_step(x, gate, state, out, slots=None, kind: str = "smooth", stream=None) -> None:
    """One position for each row of x, gate, out [rows, C]: state [pool, C] float32 is updated in place and out gets it in the
    element type.  slots: int32 [rows], the pool's row of every request, distinct (outside the pool: zeros, nothing changes)."""
    shape, dtype, device = x.shape, x.dtype, x.device
    if len(shape) != 2 or state.dim() != 2 or device.type != "cuda":
        raise ValueError("x has to be [rows, C] and state [pool, C] on a GPU")
    index = device.index
    if _current_device() != index:
        with torch.cuda.device(device):
            return recurrence_step(x, gate, state, out, slots, kind, stream)
    rows, channels = shape
    (x_stride, x_channel), (gate_stride, gate_channel), (out_stride, out_channel) = x.stride(), gate.stride(), out.stride()
    if channels != 1 and not x_channel == gate_channel == out_channel == 1:
        raise ValueError("x, gate and out: channels have to lie next to each other")
    pool = state.shape[0]
    status = _library().esrnn_recurrence_step(
        _choice(KINDS, kind, "kind"), _dtype(dtype), rows, pool, channels, x.data_ptr(), x_stride,
        _check(gate, "gate", shape, dtype, device, dense=False), gate_stride, _check_optional(slots, "slots", shape[:1], torch.int32, device),
        _check(state, "state", (pool, channels), torch.float32, device), _check(out, "out", shape, dtype, device, dense=False), out_stride,
        _raw_stream(index) if stream is None else _stream(stream, device))
    if status != ESRNN_OK:
        raise EsrnnError(status, "esrnn_recurrence_step")


class GroupNorm:
    """Group norm with activation over x [N, T, C], channels last: `groups` groups of neighbouring channels, statistics over the positions
    of a sample and a group's channels (T = 1: every position by itself), then scale and shift [C] float32, then "silu" or "none".
    lengths: int32 [N], positions that exist, or None.  Owns out, the gradients and what the reverse pass needs."""

    def __init__(self, N: int, T: int, C_: int, groups: int, activation: str = "silu", eps: float = 1e-5, dtype=None,
                 training: bool = True, device="cuda"):
        dtype = torch.float32 if dtype is None else dtype
        self.device, self.dtype, self.training = _cuda(device), dtype, training
        self._index = self.device.index
        self._lib = _library()
        self._shape = GroupNormShape(int(N), int(T), int(C_), int(groups), _choice(ACTIVATIONS, activation, "activation"), _dtype(dtype),
                                     float(eps))
        self._ref = C.byref(self._shape)
        self.workspace = torch.empty(_bytes(self._lib.esrnn_group_norm_workspace_bytes, self._ref), dtype=torch.uint8, device=self.device)
        self._size, self._channels, self._samples = torch.Size((N, T, C_)), torch.Size((C_,)), torch.Size((N,))
        self.out = torch.empty(self._size, dtype=dtype, device=self.device)
        self._out_ptr, self._workspace_ptr, self._stats_ptr = self.out.data_ptr(), self.workspace.data_ptr(), None
        self._forward_done = False
        if training:
            self.stats = torch.empty((N, groups, 2), dtype=torch.float32, device=self.device)
            self.grad_x = torch.empty(self._size, dtype=dtype, device=self.device)
            self.grad_scale, self.grad_shift = (torch.empty(C_, dtype=torch.float32, device=self.device) for _ in range(2))
            self._stats_ptr = self.stats.data_ptr()
            self._grads = [t.data_ptr() for t in (self.grad_x, self.grad_scale, self.grad_shift)]

    def _given(self, x, scale, shift, lengths):
        f = torch.float32
        return (_check(x, "x", self._size, self.dtype, self.device), _check_optional(lengths, "lengths", self._samples, torch.int32, self.device),
                _check(scale, "scale", self._channels, f, self.device), _check(shift, "shift", self._channels, f, self.device))

    def forward(self, x, scale, shift, lengths=None, stream=None):
        """out, zero past the lengths."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.forward(x, scale, shift, lengths, stream)
        _raise(self._lib.esrnn_group_norm_forward(
            self._ref, *self._given(x, scale, shift, lengths), self._out_ptr, self._stats_ptr, self._workspace_ptr,
            _raw_stream(self._index) if stream is None else _stream(stream, self.device)), "esrnn_group_norm_forward")
        self._forward_done = True
        return self.out

    def backward(self, x, scale, shift, grad_out, lengths=None, stream=None):
        """(grad_x, grad_scale, grad_shift) for the forward pass last run, which had the same x, scale, shift and lengths."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.backward(x, scale, shift, grad_out, lengths, stream)
        if not self.training or not self._forward_done:
            raise EsrnnError(4, "GroupNorm.backward")
        _raise(self._lib.esrnn_group_norm_backward(
            self._ref, *self._given(x, scale, shift, lengths), self._stats_ptr,
            _check(grad_out, "grad_out", self._size, self.dtype, self.device), *self._grads, self._workspace_ptr,
            _raw_stream(self._index) if stream is None else _stream(stream, self.device)), "esrnn_group_norm_backward")
        return self.grad_x, self.grad_scale, self.grad_shift


class AdamW:
    """One AdamW update of many tensors at once: params float32, grads float32, bfloat16 or float16 tensors of the same sizes whose
    contents the caller renews in place, optionally copies (bfloat16 or float16) that get the updated parameters.  weight_decay:
    one number, or one for each tensor.  clip_norm > 0 clips the gradient by its global norm, leaves the norm in grad_norm, and
    changes nothing where the norm is not finite.

    state_bits 32: m, v float32.  8: m and r = sqrt(v) float8_e4m3fn in units of m_scale, r_scale (float32, one for 256
    elements), rounded at random with seed.  All flat, a tensor's elements from a multiple of 256 on (offsets), zero at the start.
    The tensors are kept referenced; lr and the other hyper-parameters are plain attributes and may change between steps.  Another list of tensors is
    another AdamW: its table takes 0.1 ms for 24 tensors, 0.7 ms for 400, and its moments begin at zero.

    A step captured into a graph keeps its number: replays repeat its bias correction and, with 8-bit moments, its random bits, which then no
    longer keep the mean.  Leave step() out of graphs that are replayed from step to step."""

    def __init__(self, params: Sequence, grads: Sequence, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                 weight_decay=0.01, clip_norm: float = 0.0, state_bits: int = 32, seed: int = 0, copies: Optional[Sequence] = None):
        self._handle = None
        params, grads = list(params), list(grads)
        copies = [None] * len(params) if copies is None else list(copies)
        decays = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * len(params)
        if not params or len({len(params), len(grads), len(copies), len(decays)}) != 1:
            raise ValueError("params, grads, copies and weight decays have to be lists of the same length, at least one")
        self.device = _cuda(params[0].device)
        self._index = self.device.index
        table = (AdamWTensor * len(params))()
        self.offsets, at = [], 0
        for i, (p, g, c, d) in enumerate(zip(params, grads, copies, decays)):
            e = table[i]
            e.param = _check(p, f"params[{i}]", p.shape, torch.float32, self.device)
            e.grad, e.grad_dtype = _check(g, f"grads[{i}]", p.shape, g.dtype, self.device), _dtype(g.dtype)
            if c is not None:
                e.copy, e.copy_dtype = _check(c, f"copies[{i}]", p.shape, c.dtype, self.device), _dtype(c.dtype)
            e.n, e.weight_decay = p.numel(), float(d)
            self.offsets.append(at)
            at += -(-p.numel() // ADAMW_BLOCK) * ADAMW_BLOCK
        self._lib, self._tensors = _library(), (params, grads, copies)
        handle = C.c_void_p()
        _raise(self._lib.esrnn_adamw_create(table, len(params), int(state_bits), C.byref(handle)), "esrnn_adamw_create")
        self._handle = handle
        n = _bytes(self._lib.esrnn_adamw_state_elements, handle)
        assert n == at
        zeros = lambda size, dtype: torch.zeros(size, dtype=dtype, device=self.device)  # noqa: E731
        self.v = self.r = self.m_scale = self.r_scale = None
        if state_bits == 32:
            self.m, self.v = zeros(n, torch.float32), zeros(n, torch.float32)
        else:
            self.m, self.r = (zeros(n, torch.uint8).view(torch.float8_e4m3fn) for _ in range(2))
            self.m_scale, self.r_scale = zeros(n // ADAMW_BLOCK, torch.float32), zeros(n // ADAMW_BLOCK, torch.float32)
        self.grad_norm = zeros(1, torch.float32)
        self.workspace = torch.empty(_bytes(self._lib.esrnn_adamw_workspace_bytes, handle), dtype=torch.uint8, device=self.device)
        self.lr, self.beta1, self.beta2, self.eps, self.clip_norm, self.seed = lr, beta1, beta2, eps, clip_norm, int(seed)
        self._states = [None if t is None else t.data_ptr() for t in (self.m, self.v, self.r, self.m_scale, self.r_scale, self.grad_norm,
                                                                      self.workspace)]
        with torch.cuda.device(self.device):
            _raise(self._lib.esrnn_adamw_bind(handle, self._states[-1], _raw_stream(self._index)), "esrnn_adamw_bind")

    def step(self, step: int, stream=None) -> None:
        """Update number `step`, from 1 on.  (The first one on another stream than the constructor's has to be ordered behind it.)"""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.step(step, stream)
        if self._handle is None:
            raise EsrnnError(1, "AdamW.step after close")
        opt = AdamWConfig(self.lr, self.beta1, self.beta2, self.eps, self.clip_norm, self.seed & 0xFFFFFFFF)
        _raise(self._lib.esrnn_adamw_update(
            self._handle, C.byref(opt), int(step), *self._states,
            _raw_stream(self._index) if stream is None else _stream(stream, self.device)), "esrnn_adamw_update")

    def close(self) -> None:
        if self._handle is not None:
            self._lib.esrnn_adamw_destroy(self._handle)
            self._handle = None

    def __del__(self):
        self.close()
