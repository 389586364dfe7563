"""Host-side checks of the layer operators (include/esrnn_layers.h) that need no GPU: exported symbols, structures of the binding, sizes, and the
refusals of every call, which come before anything is launched."""
import ctypes as C
import os
import re

import pytest

from paper_1907_03329_amd import binding, layers

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, CONFIG, WORKSPACE, ORDER = 0, 1, 2, 3, 4
# addresses that are looked at, never followed
P, WS = C.c_void_p(1 << 20), C.c_void_p(1 << 20)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1907_03329_amd import build
        build.build()
    return layers._library()


def declared():
    text = open(os.path.join(ROOT, "include", "esrnn_layers.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_every_declared_symbol_is_exported_and_has_a_signature(lib):
    names = sorted(set(re.findall(r"\b(esrnn_[a-z_]+)\s*\(", declared())))
    assert len(names) == 14
    for n in names:
        assert getattr(lib, n).argtypes is not None, n
        params = re.search(rf"\b{n}\s*\(([^)]*)\)", declared()).group(1)
        assert len(getattr(lib, n).argtypes) == params.count(",") + 1, n


def test_structures_have_the_headers_layout():
    assert C.sizeof(layers.RecurrenceShape) == 24 + 6 * 2 * 8       # five int32, padding, six pairs of int64
    assert layers.RecurrenceShape.x_stride.offset == 24
    assert C.sizeof(layers.GroupNormShape) == 28
    assert C.sizeof(layers.AdamWTensor) == 48
    assert C.sizeof(layers.AdamWConfig) == 48


def recurrence(B=2, T=300, C_=64, kind=0, dtype=0, **strides):
    s = layers.RecurrenceShape()
    s.B, s.T, s.C, s.kind, s.dtype = B, T, C_, kind, dtype
    for name in ("x_stride", "gate_stride", "out_stride", "grad_out_stride", "grad_x_stride", "grad_gate_stride"):
        v = strides.get(name, (T * C_, C_))
        getattr(s, name)[0], getattr(s, name)[1] = v
    return s


def size_of(fn, *args):
    n = C.c_size_t()
    assert fn(*args, C.byref(n)) == OK
    return n.value


def test_recurrence_sizes(lib):
    saved = lambda **kw: size_of(lib.esrnn_recurrence_saved_bytes, C.byref(recurrence(**kw)))  # noqa: E731
    work = lambda **kw: size_of(lib.esrnn_recurrence_workspace_bytes, C.byref(recurrence(**kw)))  # noqa: E731
    # a state of every channel for at least every 256 positions, and no more than for every 8
    for T in (1, 8, 9, 100, 1000, 100000):
        for B, C_ in ((1, 1), (3, 70), (400, 100)):
            assert 4 * B * C_ * -(-T // 256) <= saved(B=B, T=T, C_=C_) <= 4 * B * C_ * -(-T // 8)
    # few channels and many positions: the maps of the blocks (two floats a channel and block of 128), of groups of them, and tickets
    n = work(B=1, T=1 << 17, C_=64)
    assert 8 * 64 * 1024 < n < 8 * 64 * 1024 * 1.1 + 4096
    assert work(B=400, T=100, C_=64) == 256


@pytest.mark.parametrize("bad", [dict(B=0), dict(T=0), dict(C_=0), dict(B=-1), dict(kind=2), dict(dtype=3), dict(dtype=-1), dict(B=1 << 23, C_=64),
                                 dict(C_=1 << 25), dict(T=(1 << 30) + 1)])
def test_recurrence_shapes_that_are_refused(lib, bad):
    n = C.c_size_t()
    s = recurrence(**bad)
    assert lib.esrnn_recurrence_saved_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert lib.esrnn_recurrence_workspace_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert lib.esrnn_recurrence_forward(C.byref(s), P, P, None, None, P, None, None, WS, None) == CONFIG


def test_recurrence_arguments_that_are_refused(lib):
    ok = recurrence()
    n = C.c_size_t()
    assert lib.esrnn_recurrence_saved_bytes(None, C.byref(n)) == NULL and lib.esrnn_recurrence_saved_bytes(C.byref(ok), None) == NULL
    forward = [C.byref(ok), P, P, None, None, P, None, None, WS, None]
    for i in (0, 1, 2, 5, 8):
        assert lib.esrnn_recurrence_forward(*[None if j == i else a for j, a in enumerate(forward)]) == NULL
    backward = [C.byref(ok), P, P, None, P, P, None, P, P, None, WS, None]
    for i in (0, 1, 2, 4, 5, 7, 8, 10):
        assert lib.esrnn_recurrence_backward(*[None if j == i else a for j, a in enumerate(backward)]) == NULL
    assert lib.esrnn_recurrence_forward(C.byref(ok), P, P, None, None, P, None, None, C.c_void_p((1 << 20) + 64), None) == WORKSPACE
    for odd in (C.c_void_p((1 << 20) + 2), C.c_void_p((1 << 20) + 1)):       # fp32 elements at an address that is none of a float
        assert lib.esrnn_recurrence_forward(C.byref(ok), odd, P, None, None, P, None, None, WS, None) == CONFIG
        assert lib.esrnn_recurrence_forward(C.byref(ok), P, P, odd, None, P, None, None, WS, None) == CONFIG
        assert lib.esrnn_recurrence_forward(C.byref(ok), P, P, None, odd, P, None, None, WS, None) == CONFIG
    # outputs that overlap themselves, strides that are negative or leave every address space
    for name, stride in (("out_stride", (0, 64)), ("out_stride", (300 * 64, 63)), ("out_stride", (64, 64)), ("x_stride", (-1, 64)),
                         ("gate_stride", (300 * 64, -64)), ("x_stride", (1 << 41, 64)), ("x_stride", (64, 1 << 40))):
        s = recurrence(**{name: stride})
        assert lib.esrnn_recurrence_forward(C.byref(s), P, P, None, None, P, None, None, WS, None) == CONFIG
    for name, stride in (("grad_x_stride", (0, 64)), ("grad_gate_stride", (300 * 64, 32)), ("grad_out_stride", (-64, 64))):
        s = recurrence(**{name: stride})
        assert lib.esrnn_recurrence_backward(C.byref(s), P, P, None, P, P, None, P, P, None, WS, None) == CONFIG


def test_single_positions_that_are_refused(lib):
    def step(kind=0, dtype=0, rows=2, pool=4, C_=8, x=P, xs=8, gate=P, gs=8, slots=P, state=P, out=P, os_=8):
        return lib.esrnn_recurrence_step(kind, dtype, rows, pool, C_, x, xs, gate, gs, slots, state, out, os_, None)
    assert step(rows=0) == OK and step(rows=0, x=None, gate=None, state=None, out=None) == OK       # no work
    for bad in (dict(kind=2), dict(dtype=5), dict(rows=-1), dict(C_=0), dict(pool=-1), dict(slots=None, rows=5), dict(xs=-8), dict(os_=7),
                dict(gs=1 << 41), dict(state=C.c_void_p(2 + (1 << 20)))):
        assert step(**bad) == CONFIG, bad
    for name in ("x", "gate", "state", "out"):
        assert step(**{name: None}) == NULL


def norm(N=2, T=30, C_=64, G=4, act=1, dtype=0, eps=1e-5):
    return layers.GroupNormShape(N, T, C_, G, act, dtype, eps)


@pytest.mark.parametrize("bad", [dict(N=0), dict(T=0), dict(C_=0), dict(G=0), dict(G=3), dict(G=128), dict(act=2), dict(dtype=3), dict(eps=0.0),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(N=1 << 20, T=1 << 12), dict(N=1 << 23),
                                 dict(N=1 << 20, C_=64, G=64), dict(C_=(1 << 20) + 4)])
def test_norm_shapes_that_are_refused(lib, bad):
    n = C.c_size_t()
    s = norm(**bad)
    assert lib.esrnn_group_norm_workspace_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert lib.esrnn_group_norm_forward(C.byref(s), P, None, P, P, P, None, WS, None) == CONFIG
    assert lib.esrnn_group_norm_backward(C.byref(s), P, None, P, P, P, P, P, P, P, WS, None) == CONFIG


def test_norm_arguments_that_are_refused(lib):
    ok = norm()
    assert size_of(lib.esrnn_group_norm_workspace_bytes, C.byref(ok)) % 256 == 0
    forward = [C.byref(ok), P, None, P, P, P, None, WS, None]
    for i in (0, 1, 3, 4, 5, 7):
        assert lib.esrnn_group_norm_forward(*[None if j == i else a for j, a in enumerate(forward)]) == NULL
    backward = [C.byref(ok), P, None, P, P, P, P, P, P, P, WS, None]
    for i in (0, 1, 3, 4, 5, 6, 7, 8, 9, 10):
        assert lib.esrnn_group_norm_backward(*[None if j == i else a for j, a in enumerate(backward)]) == NULL
    odd = C.c_void_p((1 << 20) + 2)
    assert lib.esrnn_group_norm_forward(C.byref(ok), odd, None, P, P, P, None, WS, None) == CONFIG
    assert lib.esrnn_group_norm_forward(C.byref(ok), P, None, P, P, P, None, odd, None) == WORKSPACE


def test_norm_workspaces_stay_small(lib):
    """Less than the input, but for a few rows of partial sums: the reverse pass leaves a row of sums for a sample or a chunk, not for a position."""
    for N, T, C_, G in ((16384, 1, 2048, 16), (1 << 20, 1, 64, 4), (6, 16384, 256, 32), (512, 72, 64, 8), (4, 100000, 512, 8)):
        n = size_of(lib.esrnn_group_norm_workspace_bytes, C.byref(norm(N, T, C_, G)))
        assert n <= N * T * C_ * 4 / 8 + (1 << 23), (N, T, C_, G, n)


def tensors(**kw):
    t = layers.AdamWTensor(1 << 20, 1 << 20, None, 1000, 0.01, 0, 0)
    for k, v in kw.items():
        setattr(t, k, v)
    return (layers.AdamWTensor * 2)(layers.AdamWTensor(1 << 20, 1 << 20, None, 5, 0.0, 1, 0), t)


@pytest.mark.parametrize("bad,status", [(dict(param=None), NULL), (dict(grad=None), NULL), (dict(n=0), CONFIG), (dict(n=-1), CONFIG),
                                        (dict(weight_decay=-0.1), CONFIG), (dict(weight_decay=float("nan")), CONFIG),
                                        (dict(grad_dtype=3), CONFIG), (dict(copy=1 << 20, copy_dtype=0), CONFIG), (dict(param=(1 << 20) + 2), CONFIG),
                                        (dict(grad=(1 << 20) + 1), CONFIG), (dict(n=1 << 39), CONFIG)])
def test_tensor_lists_that_are_refused(lib, bad, status):
    h = C.c_void_p(5)
    assert lib.esrnn_adamw_create(tensors(**bad), 2, 32, C.byref(h)) == status
    assert not h.value


def test_adamw_handles(lib):
    h, n = C.c_void_p(), C.c_size_t()
    assert lib.esrnn_adamw_create(None, 1, 32, C.byref(h)) == NULL and lib.esrnn_adamw_create(tensors(), 2, 32, None) == NULL
    assert lib.esrnn_adamw_create(tensors(), 0, 32, C.byref(h)) == CONFIG and lib.esrnn_adamw_create(tensors(), 2, 16, C.byref(h)) == CONFIG
    assert lib.esrnn_adamw_destroy(None) == NULL
    for bits in (32, 8):
        assert lib.esrnn_adamw_create(tensors(), 2, bits, C.byref(h)) == OK
        assert size_of(lib.esrnn_adamw_state_elements, h) == 256 + 1024
        assert size_of(lib.esrnn_adamw_workspace_bytes, h) % 256 == 0
        opt = layers.AdamWConfig(1e-3, 0.9, 0.999, 1e-8, 0.0, 0)
        call = lambda o=opt, step=1, m=P, v=P, r=P, ms=P, rs=P, ws=WS: lib.esrnn_adamw_update(h, C.byref(o), step, m, v, r, ms, rs, None, ws, None)  # noqa: E731
        assert call() == ORDER                  # no bind before
        assert call(m=None) == NULL and call(ws=None) == NULL
        assert (call(v=None) == NULL) == (bits == 32)
        assert (call(r=None) == NULL) == (bits == 8) and (call(rs=None) == NULL) == (bits == 8)
        assert call(step=0) == CONFIG
        for kw in (dict(beta1=1.0), dict(beta2=1.5), dict(beta1=-0.1), dict(lr=-1.0), dict(lr=float("inf")), dict(eps=float("nan")),
                   dict(clip_norm=float("nan"))):
            o = layers.AdamWConfig(1e-3, 0.9, 0.999, 1e-8, 0.0, 0)
            for k, v in kw.items():
                setattr(o, k, v)
            assert call(o) == CONFIG, kw
        assert call(m=C.c_void_p((1 << 20) + 2)) == CONFIG
        assert lib.esrnn_adamw_bind(h, C.c_void_p((1 << 20) + 8), None) == WORKSPACE and lib.esrnn_adamw_bind(h, None, None) == NULL
        assert lib.esrnn_adamw_destroy(h) == OK

