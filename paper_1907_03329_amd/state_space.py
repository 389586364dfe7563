"""Thin ctypes binding of the operators of a selective state space layer (C ABI in include/esrnn_state_space.h): short causal convolution,
selective scan, and the norms around a block with its gate and residual.

Argument marshalling only, as in layers.py: the classes own the buffers of a layer, every call runs in the library's kernels on the
current stream of the tensors' device (or the one given), and a failed call raises EsrnnError.  There is no fallback.
Tensors that a call names have to live until the stream has run it, as with any work of torch on that stream.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import layers
from .binding import EsrnnError, load_library
from .layers import ACTIVATIONS, _bytes, _check, _check_optional, _choice, _cuda, _dtype, _raise, _stream

DELTAS = {"softplus": 0, "given": 1}
GATES = {"none": 0, "before": 1, "after": 2}


def _strides(*names):
    return [(name + "_stride", C.c_int64 * 2) for name in names]


class ConvolutionShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("B", "T", "C", "K", "activation", "dtype")] + _strides("x", "out", "grad_out", "grad_x")


class ConvolutionStepShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("rows", "pool", "C", "K", "activation", "dtype")] + [
        (name, C.c_int64) for name in ("x_stride", "out_stride")]


class SelectiveShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("B", "T", "C", "N", "G", "delta_kind", "dtype")] + _strides(
        "x", "delta", "b", "c", "out", "grad_out", "grad_x", "grad_delta", "grad_b", "grad_c")


class SelectiveGrads(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("x", "delta", "b", "c", "A", "D", "bias", "initial")]


class SelectiveStepShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("rows", "pool", "C", "N", "G", "delta_kind", "dtype")] + [
        (name, C.c_int64) for name in ("x_stride", "delta_stride", "b_stride", "c_stride", "out_stride")]


class BlockNormShape(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("rows", "C", "gate", "dtype", "stream_dtype")] + [("eps", C.c_float)] + [
        (name + "_stride", C.c_int64) for name in ("y", "gate", "residual", "sum", "out", "grad_out", "grad_sum", "grad_y", "grad_gate", "grad_residual")]


class BlockNormOperands(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("y", "gate", "residual", "exists", "post_weight", "scale", "pre_weight")]


class BlockNormGrads(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("y", "gate", "residual", "post_weight", "scale", "pre_weight")]


_lib = None


def _library():
    """The library with the signatures of include/esrnn_state_space.h."""
    global _lib
    if _lib is not None:
        return _lib
    lib = load_library()
    vp, size = C.c_void_p, C.POINTER(C.c_size_t)
    conv, select, block = C.POINTER(ConvolutionShape), C.POINTER(SelectiveShape), C.POINTER(BlockNormShape)
    operands = C.POINTER(BlockNormOperands)
    for name, args in {
        "esrnn_convolution_workspace_bytes": [conv, size],
        "esrnn_convolution_forward": [conv] + [vp] * 8,
        "esrnn_convolution_backward": [conv] + [vp] * 13,
        "esrnn_convolution_step": [C.POINTER(ConvolutionStepShape)] + [vp] * 7,
        "esrnn_selective_workspace_bytes": [select, C.c_int32, size],
        "esrnn_selective_saved_bytes": [select, size],
        "esrnn_selective_forward": [select] + [vp] * 14,
        "esrnn_selective_backward": [select] + [vp] * 11 + [C.POINTER(SelectiveGrads), vp, vp],
        "esrnn_selective_step": [C.POINTER(SelectiveStepShape)] + [vp] * 11,
        "esrnn_block_norm_workspace_bytes": [block, size],
        "esrnn_block_norm_forward": [block, operands] + [vp] * 4,
        "esrnn_block_norm_backward": [block, operands] + [vp] * 3 + [C.POINTER(BlockNormGrads), vp, vp],
    }.items():
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, C.c_int
    _lib = lib
    return lib


def _of_device(stream, index, device):
    """The stream of a call as the library takes it."""
    return layers._raw_stream(index) if stream is None else _stream(stream, device)


def _positions(t, name, size, dtype, device, field, time_major) -> int:
    """The address of a tensor over sequences and positions; its strides go into `field`."""
    at = _check(t, name, size, dtype, device, dense=False)
    stride = t.stride()
    if stride[-1] != 1 and size[-1] != 1:
        raise ValueError(f"{name}: channels have to lie next to each other")
    if len(size) == 4 and stride[2] != size[3] and size[2] != 1:
        raise ValueError(f"{name}: groups have to lie next to each other")
    field[0], field[1] = (stride[1], stride[0]) if time_major else (stride[0], stride[1])
    return at


def _row_stride(t, name):
    row, channel = t.stride()
    if channel != 1 and t.shape[1] != 1:
        raise ValueError(f"{name}: channels have to lie next to each other")
    return row


def _remembered(shapes, make, *values):
    """The shape of a call of single positions: a structure made once for each set of values (a few for a server's batch sizes)."""
    shape = shapes.get(values)
    if shape is None:
        if len(shapes) >= 256:
            shapes.clear()
        shape = shapes[values] = C.byref(make(*values))
    return shape


def _held(layer, t, name, size, dtype, own, stream):
    """The address of states that a call reads: of a copy, if they are the layer's `own` that the call overwrites."""
    if t is None:
        return None
    at = _check(t, name, size, dtype, layer.device)
    if at != own:
        return at
    kept = layer._carried.get(name)
    if kept is None:
        kept = layer._carried[name] = torch.empty_like(t)
    with torch.cuda.stream(stream):     # (None: the current one)
        kept.copy_(t)
    return kept.data_ptr()


class ShortConvolution:
    """out_t = act(bias + sum_j weight[:, j] x_{t-K+1+j}) over sequences of up to T positions, every one of C channels with K taps of its own, 2 to 8.

    Tensors are [B, T, C], with time_major [T, B, C]; x, grad_out (and grad_x, where the caller gives it) may be strided in any way that
    keeps channels next to each other.  weight: float32 [C, K], bias float32 [C] or None.  lengths: int32 [B], positions that exist.
    initial: [B, K - 1, C] in the element type, the inputs before the first position, oldest first, or None (zero).  grad_last: float32.
    Owns out, last, the gradients and the workspace, all overwritten by the next call; last may be that call's initial, and grad_initial
    the next reverse pass's grad_last (they are copied before)."""

    def __init__(self, B: int, T: int, C_: int, taps: int = 4, activation: str = "silu", dtype=None, time_major: bool = False,
                 training: bool = True, device="cuda"):
        dtype = torch.float32 if dtype is None else dtype
        self.device, self.dtype, self.time_major, self.training = _cuda(device), dtype, time_major, training
        self._index, self._lib = self.device.index, _library()
        s = ConvolutionShape()
        s.B, s.T, s.C, s.K, s.activation, s.dtype = int(B), int(T), int(C_), int(taps), _choice(ACTIVATIONS, activation, "activation"), _dtype(dtype)
        self._shape, self._ref = s, C.byref(s)
        workspace = _bytes(self._lib.esrnn_convolution_workspace_bytes, self._ref)
        self._size, self._window = torch.Size((T, B, C_) if time_major else (B, T, C_)), torch.Size((B, taps - 1, C_))
        self._taps, self._channels, self._sequences = torch.Size((C_, taps)), torch.Size((C_,)), torch.Size((B,))
        empty = lambda size, dt=torch.float32: torch.empty(size, dtype=dt, device=self.device)  # noqa: E731
        self.out, self.last, self._carried, self._own_first = empty(self._size, dtype), empty(self._window, dtype), {}, False
        self._out_ptr, self._last_ptr = self.out.data_ptr(), self.last.data_ptr()
        self._positions(self.out, "out", s.out_stride)
        if training:
            self.workspace = empty(workspace, torch.uint8)
            self.grad_x, self.grad_initial = empty(self._size, dtype), empty(self._window)
            self.grad_weight, self.grad_bias = empty(self._taps), empty(self._channels)
            self._sums = [t.data_ptr() for t in (self.grad_weight, self.grad_bias, self.grad_initial, self.workspace)]

    def _positions(self, t, name, field):
        return _positions(t, name, self._size, self.dtype, self.device, field, self.time_major)

    def _given(self, x, weight, bias, lengths):
        f, d = torch.float32, self.device
        return (self._positions(x, "x", self._shape.x_stride), _check_optional(lengths, "lengths", self._sequences, torch.int32, d),
                _check(weight, "weight", self._taps, f, d), _check_optional(bias, "bias", self._channels, f, d))

    def forward(self, x, weight, bias=None, lengths=None, initial=None, stream=None):
        """(out, last): out zero past the lengths, and the last K - 1 inputs of every sequence."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.forward(x, weight, bias, lengths, initial, stream)
        given = self._given(x, weight, bias, lengths)
        to = _of_device(stream, self._index, self.device)
        first = _held(self, initial, "initial", self._window, self.dtype, self._last_ptr, stream)
        _raise(self._lib.esrnn_convolution_forward(self._ref, *given, first, self._out_ptr, self._last_ptr, to), "esrnn_convolution_forward")
        self._own_first = initial is not None and initial.data_ptr() == self._last_ptr
        return self.out, self.last

    def backward(self, x, weight, grad_out, bias=None, lengths=None, initial=None, grad_last=None, grad_x=None, stream=None):
        """(grad_x, grad_weight, grad_bias, grad_initial) for the operands of a forward pass.  `initial` may be the layer's own `last` if that was what the
        forward pass last run was given: what it held then."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.backward(x, weight, grad_out, bias, lengths, initial, grad_last, grad_x, stream)
        if not self.training:
            raise EsrnnError(4, "ShortConvolution.backward")
        grad_x, s = self.grad_x if grad_x is None else grad_x, self._shape
        given = self._given(x, weight, bias, lengths)
        d_ptr, gx_ptr = self._positions(grad_out, "grad_out", s.grad_out_stride), self._positions(grad_x, "grad_x", s.grad_x_stride)
        first = _check_optional(initial, "initial", self._window, self.dtype, self.device)
        if first == self._last_ptr:
            if not self._own_first:
                raise ValueError("initial is what the forward pass has written to the layer's last")
            first = self._carried["initial"].data_ptr()
        to = _of_device(stream, self._index, self.device)
        gw, gb, gi, workspace = self._sums
        _raise(self._lib.esrnn_convolution_backward(
            self._ref, *given, first, d_ptr, _held(self, grad_last, "grad_last", self._window, torch.float32, gi, stream), gx_ptr, gw, gb, gi, workspace, to),
            "esrnn_convolution_backward")
        return grad_x, self.grad_weight, self.grad_bias, self.grad_initial


_convolution_shapes, _selective_shapes = {}, {}


def convolution_step(x, weight, state, out, bias=None, slots=None, activation: str = "silu", stream=None) -> None:
    """One position for each row of x and out [rows, C]: state [pool, K - 1, C] in the element type, the inputs before, oldest first, is moved on in
    place.  slots: int32 [rows], the pool's row of every request, distinct (outside the pool: zeros, nothing changes)."""
    shape, dtype, device = x.shape, x.dtype, x.device
    if len(shape) != 2 or state.dim() != 3 or device.type != "cuda":
        raise ValueError("x has to be [rows, C] and state [pool, K - 1, C] on a GPU")
    index = device.index
    if layers._current_device() != index:
        with torch.cuda.device(device):
            return convolution_step(x, weight, state, out, bias, slots, activation, stream)
    (rows, channels), (pool, past, _) = shape, state.shape
    s = _remembered(_convolution_shapes, ConvolutionStepShape, rows, pool, channels, past + 1, _choice(ACTIVATIONS, activation, "activation"), _dtype(dtype),
                    _row_stride(x, "x"), _row_stride(out, "out"))
    f = torch.float32
    _raise(_library().esrnn_convolution_step(
        s, x.data_ptr(), _check(weight, "weight", (channels, past + 1), f, device), _check_optional(bias, "bias", (channels,), f, device),
        _check_optional(slots, "slots", shape[:1], torch.int32, device), _check(state, "state", (pool, past, channels), dtype, device),
        _check(out, "out", shape, dtype, device, dense=False), _of_device(stream, index, device)), "esrnn_convolution_step")


class SelectiveScan:
    """h_t = exp(d_t A) h_{t-1} + d_t x_t b_t, out_t = c_t h_t + D x_t over sequences of up to T positions: C channels of N states each, 1 to 64, with
    d = softplus(delta + bias) or, with delta_kind "given", delta + bias.  b and c belong to `groups` groups of neighbouring channels.

    x, delta and gradients of them are [B, T, C], b and c [B, T, groups, N], with time_major [T, B, ..]; all may be strided in any way that keeps
    channels, and groups and states, next to each other.  A: float32 [C, N], used as it is; D, bias: float32 [C] or None (zero).
    lengths: int32 [B], positions that exist; initial, grad_last: float32 [B, C, N] or None (zero).
    Owns out, last, the gradients and what the reverse pass needs, all overwritten by the next call; last may be that call's initial, and
    grad_initial the next reverse pass's grad_last (they are copied before)."""

    def __init__(self, B: int, T: int, C_: int, N: int, groups: int = 1, delta_kind: str = "softplus", dtype=None, time_major: bool = False,
                 training: bool = True, device="cuda"):
        dtype = torch.float32 if dtype is None else dtype
        self.device, self.dtype, self.time_major, self.training = _cuda(device), dtype, time_major, training
        self._index, self._lib = self.device.index, _library()
        s = SelectiveShape()
        s.B, s.T, s.C, s.N, s.G = int(B), int(T), int(C_), int(N), int(groups)
        s.delta_kind, s.dtype = _choice(DELTAS, delta_kind, "delta_kind"), _dtype(dtype)
        self._shape, self._ref = s, C.byref(s)
        workspace = _bytes(self._lib.esrnn_selective_workspace_bytes, self._ref, int(training))
        saved = _bytes(self._lib.esrnn_selective_saved_bytes, self._ref)
        lead = (T, B) if time_major else (B, T)
        self._size, self._shared, self._states = torch.Size((*lead, C_)), torch.Size((*lead, groups, N)), torch.Size((B, C_, N))
        self._rates, self._channels, self._sequences = torch.Size((C_, N)), torch.Size((C_,)), torch.Size((B,))
        empty = lambda size, dt=torch.float32: torch.empty(size, dtype=dt, device=self.device)  # noqa: E731
        self.workspace, self.out, self.last = empty(workspace, torch.uint8), empty(self._size, dtype), empty(self._states)
        self._workspace_ptr, self._out_ptr, self._last_ptr = (t.data_ptr() for t in (self.workspace, self.out, self.last))
        self._wide(self.out, "out", s.out_stride)
        self._forward_done, self._saved_ptr, self._carried = False, None, {}
        if training:
            self.saved = empty(saved // 4)
            self._saved_ptr = self.saved.data_ptr()
            self.grad_x, self.grad_delta = empty(self._size, dtype), empty(self._size, dtype)
            self.grad_b, self.grad_c = empty(self._shared, dtype), empty(self._shared, dtype)
            self.grad_A, self.grad_D, self.grad_bias, self.grad_initial = empty(self._rates), empty(self._channels), empty(self._channels), empty(self._states)
            self._grads = SelectiveGrads(A=self.grad_A.data_ptr(), D=self.grad_D.data_ptr(), bias=self.grad_bias.data_ptr(), initial=self.grad_initial.data_ptr())
            self._grads_ref = C.byref(self._grads)

    def _wide(self, t, name, field):
        return _positions(t, name, self._size, self.dtype, self.device, field, self.time_major)

    def _narrow(self, t, name, field):
        return _positions(t, name, self._shared, self.dtype, self.device, field, self.time_major)

    def _given(self, x, delta, A, b, c, D, bias, lengths):
        s, f, d = self._shape, torch.float32, self.device
        return (self._wide(x, "x", s.x_stride), self._wide(delta, "delta", s.delta_stride), _check(A, "A", self._rates, f, d),
                self._narrow(b, "b", s.b_stride), self._narrow(c, "c", s.c_stride), _check_optional(D, "D", self._channels, f, d),
                _check_optional(bias, "bias", self._channels, f, d), _check_optional(lengths, "lengths", self._sequences, torch.int32, d))

    def forward(self, x, delta, A, b, c, D=None, bias=None, lengths=None, initial=None, stream=None):
        """(out, last): out in the element type, zero past the lengths, and the last state of every sequence in float32."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.forward(x, delta, A, b, c, D, bias, lengths, initial, stream)
        given = self._given(x, delta, A, b, c, D, bias, lengths)
        to = _of_device(stream, self._index, self.device)
        _raise(self._lib.esrnn_selective_forward(
            self._ref, *given, _held(self, initial, "initial", self._states, torch.float32, self._last_ptr, stream), self._out_ptr, self._last_ptr,
            self._saved_ptr, self._workspace_ptr, to), "esrnn_selective_forward")
        self._forward_done = True
        return self.out, self.last

    def backward(self, x, delta, A, b, c, grad_out, D=None, bias=None, lengths=None, grad_last=None, grad_x=None, grad_delta=None, grad_b=None,
                 grad_c=None, stream=None):
        """(grad_x, grad_delta, grad_A, grad_b, grad_c, grad_D, grad_bias, grad_initial) for the forward pass last run, which had the same operands."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.backward(x, delta, A, b, c, grad_out, D, bias, lengths, grad_last, grad_x, grad_delta, grad_b, grad_c, stream)
        if not self.training or not self._forward_done:
            raise EsrnnError(4, "SelectiveScan.backward")
        own = (self.grad_x, self.grad_delta, self.grad_b, self.grad_c)
        grad_x, grad_delta, grad_b, grad_c = (mine if t is None else t for t, mine in zip((grad_x, grad_delta, grad_b, grad_c), own))
        given, s, g = self._given(x, delta, A, b, c, D, bias, lengths), self._shape, self._grads
        d_ptr = self._wide(grad_out, "grad_out", s.grad_out_stride)
        g.x, g.delta = self._wide(grad_x, "grad_x", s.grad_x_stride), self._wide(grad_delta, "grad_delta", s.grad_delta_stride)
        g.b, g.c = self._narrow(grad_b, "grad_b", s.grad_b_stride), self._narrow(grad_c, "grad_c", s.grad_c_stride)
        to = _of_device(stream, self._index, self.device)
        _raise(self._lib.esrnn_selective_backward(
            self._ref, *given, self._saved_ptr, d_ptr, _held(self, grad_last, "grad_last", self._states, torch.float32, g.initial, stream),
            self._grads_ref, self._workspace_ptr, to), "esrnn_selective_backward")
        return grad_x, grad_delta, self.grad_A, grad_b, grad_c, self.grad_D, self.grad_bias, self.grad_initial


def selective_step(x, delta, A, b, c, state, out, D=None, bias=None, slots=None, delta_kind: str = "softplus", stream=None) -> None:
    """One position for each row of x, delta, out [rows, C] and b, c [rows, groups, N]: state [pool, C, N] float32 is updated in place.  slots: int32
    [rows], the pool's row of every request, distinct (outside the pool: zeros, nothing changes)."""
    shape, dtype, device = x.shape, x.dtype, x.device
    if len(shape) != 2 or state.dim() != 3 or b.dim() != 3 or device.type != "cuda":
        raise ValueError("x has to be [rows, C], b [rows, groups, N] and state [pool, C, N] on a GPU")
    index = device.index
    if layers._current_device() != index:
        with torch.cuda.device(device):
            return selective_step(x, delta, A, b, c, state, out, D, bias, slots, delta_kind, stream)
    (rows, channels), (pool, _, N), groups = shape, state.shape, b.shape[1]
    f, shared = torch.float32, (rows, groups, N)
    for t, name in ((b, "b"), (c, "c")):
        _check(t, name, shared, dtype, device, dense=False)
        if (t.stride(2) != 1 and N != 1) or (t.stride(1) != N and groups != 1):
            raise ValueError(f"{name}: groups and states have to lie next to each other")
    s = _remembered(_selective_shapes, SelectiveStepShape, rows, pool, channels, N, groups, _choice(DELTAS, delta_kind, "delta_kind"), _dtype(dtype),
                    _row_stride(x, "x"), _row_stride(delta, "delta"), b.stride(0), c.stride(0), _row_stride(out, "out"))
    _raise(_library().esrnn_selective_step(
        s, x.data_ptr(), _check(delta, "delta", shape, dtype, device, dense=False), _check(A, "A", (channels, N), f, device), b.data_ptr(),
        c.data_ptr(), _check_optional(D, "D", (channels,), f, device), _check_optional(bias, "bias", (channels,), f, device),
        _check_optional(slots, "slots", shape[:1], torch.int32, device), _check(state, "state", (pool, channels, N), f, device),
        _check(out, "out", shape, dtype, device, dense=False), _of_device(stream, index, device)), "esrnn_selective_step")


class BlockNorm:
    """What stands between one block's result y [rows, C] and the next block's input, every row by itself:

        v = y silu(gate) (gate "before") or y;   p = v / rms(v) post_weight, or v without post_weight
        e = p silu(gate) (gate "after") or p;    sum = residual + scale e (with `residual`), else scale e
        out = sum / rms(sum) pre_weight (with `pre`)

    with rms(v) = sqrt(mean(v^2) + eps).  With `residual`, sum is left in stream_dtype (the element type or float32); without `pre` it is then the
    only result, and without either, out is scale e.  Weights: float32 [C]; exists: int32 [rows], rows with 0 give zeros and add nothing to a
    gradient.  Tensors may have any stride of rows.  Owns sum, out, the gradients and what the reverse pass needs."""

    def __init__(self, rows: int, C_: int, gate: str = "none", residual: bool = True, pre: bool = True, eps: float = 1e-5, dtype=None, stream_dtype=None,
                 training: bool = True, device="cuda"):
        dtype = torch.float32 if dtype is None else dtype
        stream_dtype = dtype if stream_dtype is None else stream_dtype
        self.device, self.dtype, self.stream_dtype, self.training, self.gate = _cuda(device), dtype, stream_dtype, training, gate
        self.residual, self.pre, self._gated = bool(residual), bool(pre), gate != "none"
        self._index, self._lib = self.device.index, _library()
        s = BlockNormShape()
        s.rows, s.C, s.gate, s.dtype, s.stream_dtype, s.eps = int(rows), int(C_), _choice(GATES, gate, "gate"), _dtype(dtype), _dtype(stream_dtype), float(eps)
        self._shape, self._ref, self._in, self._out = s, C.byref(s), BlockNormOperands(), BlockNormGrads()
        self._in_ref, self._out_ref = C.byref(self._in), C.byref(self._out)
        workspace = _bytes(self._lib.esrnn_block_norm_workspace_bytes, self._ref)
        self._size, self._channels, self._rows = torch.Size((rows, C_)), torch.Size((C_,)), torch.Size((rows,))
        empty = lambda size, dt=torch.float32: torch.empty(size, dtype=dt, device=self.device)  # noqa: E731
        self.sum = empty(self._size, stream_dtype) if residual else None
        self.out = empty(self._size, dtype) if pre or not residual else None
        s.sum_stride = s.out_stride = s.grad_y_stride = s.grad_gate_stride = s.grad_residual_stride = int(C_)
        self._sum_ptr, self._result_ptr = (None if t is None else t.data_ptr() for t in (self.sum, self.out))
        self._forward_done, self._stats_ptr = False, None
        if training:
            self.workspace, self.stats = empty(workspace, torch.uint8), empty((rows, 2))
            self._stats_ptr, self._workspace_ptr = self.stats.data_ptr(), self.workspace.data_ptr()
            self.grad_y = empty(self._size, dtype)
            self.grad_gate = empty(self._size, dtype) if gate != "none" else None
            self.grad_residual = empty(self._size, stream_dtype) if residual else None
            self.grad_post_weight, self.grad_scale, self.grad_pre_weight = (empty(self._channels) for _ in range(3))
            self._out.y = self.grad_y.data_ptr()
            self._out.gate, self._out.residual = (None if t is None else t.data_ptr() for t in (self.grad_gate, self.grad_residual))

    def _row(self, t, name, dtype):
        """The address and the stride of rows."""
        return _check(t, name, self._size, dtype, self.device, dense=False), _row_stride(t, name)

    def _absent(self, t, name, wanted):
        if (t is not None) != wanted:
            raise ValueError(f"{name} has to be {'given' if wanted else 'None'}")

    def _given(self, y, gate, residual, exists, post_weight, scale, pre_weight):
        o, s, f, d, size = self._in, self._shape, torch.float32, self.device, self._channels
        if (gate is not None) != self._gated or (residual is not None) != self.residual or (pre_weight is not None) != self.pre:
            self._absent(gate, "gate", self._gated)
            self._absent(residual, "residual", self.residual)
            self._absent(pre_weight, "pre_weight", self.pre)
        o.y, s.y_stride = self._row(y, "y", self.dtype)
        if self._gated:
            o.gate, s.gate_stride = self._row(gate, "gate", self.dtype)
        if self.residual:
            o.residual, s.residual_stride = self._row(residual, "residual", self.stream_dtype)
        if self.pre:
            o.pre_weight = _check(pre_weight, "pre_weight", size, f, d)
        o.post_weight = None if post_weight is None else _check(post_weight, "post_weight", size, f, d)
        o.scale = None if scale is None else _check(scale, "scale", size, f, d)
        o.exists = None if exists is None else _check(exists, "exists", self._rows, torch.int32, d)

    def forward(self, y, gate=None, residual=None, post_weight=None, scale=None, pre_weight=None, exists=None, in_place: bool = False, stream=None):
        """(sum, out); the one that there is not is None.  in_place: sum takes the place of `residual` (not in a layer for training)."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.forward(y, gate, residual, post_weight, scale, pre_weight, exists, in_place, stream)
        if in_place and (self.training or not self.residual):
            raise ValueError("in_place needs a residual, and a layer that is not for training")
        self._given(y, gate, residual, exists, post_weight, scale, pre_weight)
        s = self._shape
        if self.residual:
            s.sum_stride = s.residual_stride if in_place else s.C
        to = _of_device(stream, self._index, self.device)
        _raise(self._lib.esrnn_block_norm_forward(self._ref, self._in_ref, self._in.residual if in_place else self._sum_ptr, self._result_ptr,
                                                  self._stats_ptr, to), "esrnn_block_norm_forward")
        self._forward_done = True
        return residual if in_place else self.sum, self.out

    def backward(self, y, grad_out=None, grad_sum=None, gate=None, residual=None, post_weight=None, scale=None, pre_weight=None, exists=None,
                 stream=None):
        """(grad_y, grad_gate, grad_residual, grad_post_weight, grad_scale, grad_pre_weight) for the forward pass last run, which had the same operands;
        None for those that it had not.  grad_out belongs to out, grad_sum to sum (None: zero)."""
        if layers._current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.backward(y, grad_out, grad_sum, gate, residual, post_weight, scale, pre_weight, exists, stream)
        if not self.training or not self._forward_done:
            raise EsrnnError(4, "BlockNorm.backward")
        self._given(y, gate, residual, exists, post_weight, scale, pre_weight)
        s, d_ptr, ds_ptr = self._shape, None, None
        self._absent(grad_out, "grad_out", self.out is not None)
        if grad_out is not None:
            d_ptr, s.grad_out_stride = self._row(grad_out, "grad_out", self.dtype)
        if grad_sum is not None:
            self._absent(grad_sum, "grad_sum", self.residual)
            ds_ptr, s.grad_sum_stride = self._row(grad_sum, "grad_sum", self.stream_dtype)
        sums = [mine if given is not None else None for mine, given in ((self.grad_post_weight, post_weight), (self.grad_scale, scale),
                                                                        (self.grad_pre_weight, pre_weight))]
        o = self._out
        o.post_weight, o.scale, o.pre_weight = (None if t is None else t.data_ptr() for t in sums)
        to = _of_device(stream, self._index, self.device)
        _raise(self._lib.esrnn_block_norm_backward(self._ref, self._in_ref, self._stats_ptr, d_ptr, ds_ptr, self._out_ref, self._workspace_ptr, to),
               "esrnn_block_norm_backward")
        return self.grad_y, self.grad_gate, self.grad_residual, *sums
