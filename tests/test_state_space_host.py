"""Host-side checks of the operators of a selective state space layer (include/esrnn_state_space.h) that need no GPU: exported symbols, structures of the
binding, sizes, and the refusals of every call, which come before anything is launched."""
import ctypes as C
import os
import re

import pytest

from paper_1907_03329_amd import binding, state_space as ss

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, CONFIG, WORKSPACE = 0, 1, 2, 3
# addresses that are looked at, never followed, far enough from each other
FAR = 1 << 44
P = [C.c_void_p(FAR * (i + 1)) for i in range(16)]
odd = lambda p, by=1: C.c_void_p(p.value + by)  # noqa: E731


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_1907_03329_amd import build
        build.build()
    return ss._library()


def declared():
    text = open(os.path.join(ROOT, "include", "esrnn_state_space.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_every_declared_symbol_is_exported_and_has_a_signature(lib):
    names = sorted(set(re.findall(r"\b(esrnn_[a-z_]+)\s*\(", declared())))
    assert len(names) == 12
    for n in names:
        assert getattr(lib, n).argtypes is not None, n
        params = re.search(rf"\b{n}\s*\(([^)]*)\)", declared()).group(1)
        assert len(getattr(lib, n).argtypes) == params.count(",") + 1, n


def test_structures_have_the_headers_layout():
    assert C.sizeof(ss.ConvolutionShape) == 24 + 4 * 16 and ss.ConvolutionShape.x_stride.offset == 24
    assert C.sizeof(ss.ConvolutionStepShape) == 40
    assert C.sizeof(ss.SelectiveShape) == 32 + 10 * 16 and ss.SelectiveShape.x_stride.offset == 32
    assert C.sizeof(ss.SelectiveStepShape) == 32 + 5 * 8
    assert C.sizeof(ss.BlockNormShape) == 24 + 10 * 8 and ss.BlockNormShape.y_stride.offset == 24
    assert C.sizeof(ss.SelectiveGrads) == 64 and C.sizeof(ss.BlockNormOperands) == 56 and C.sizeof(ss.BlockNormGrads) == 48
    for struct, name in ((ss.ConvolutionShape, "esrnn_convolution_shape"), (ss.SelectiveShape, "esrnn_selective_shape"), (ss.BlockNormShape, "esrnn_block_norm_shape"),
                         (ss.SelectiveStepShape, "esrnn_selective_step_shape"), (ss.ConvolutionStepShape, "esrnn_convolution_step_shape"),
                         (ss.SelectiveGrads, "esrnn_selective_grads"), (ss.BlockNormGrads, "esrnn_block_norm_grads"), (ss.BlockNormOperands, "esrnn_block_norm_operands")):
        body = [b for b in re.findall(r"typedef struct \{([^}]*)\}\s*(\w+);", declared()) if b[1] == name][0][0]
        names = [n for line in body.split(";") for n in re.findall(r"[*\s,](\w+)(?:\[2\])?\s*(?=,|$)", re.sub(r"^\s*(const\s+)?\w+", "", line.strip()))]
        assert names == [f[0] for f in struct._fields_], name


# ---- short causal convolution ----
def conv(B=2, T=30, C_=64, K=4, act=1, dtype=0, **strides):
    s = ss.ConvolutionShape()
    s.B, s.T, s.C, s.K, s.activation, s.dtype = B, T, C_, K, act, dtype
    for name in ("x_stride", "out_stride", "grad_out_stride", "grad_x_stride"):
        getattr(s, name)[0], getattr(s, name)[1] = strides.get(name, (T * C_, C_))
    return s


def conv_forward(lib, s, x=P[0], lengths=None, weight=P[1], bias=P[2], initial=P[3], out=P[4], last=P[5]):
    return lib.esrnn_convolution_forward(C.byref(s) if s else None, x, lengths, weight, bias, initial, out, last, None)


def conv_backward(lib, s, x=P[0], lengths=None, weight=P[1], bias=P[2], initial=P[3], d=P[6], dlast=P[7], gx=P[8], gw=P[9], gb=P[10], gi=P[11], ws=P[12]):
    return lib.esrnn_convolution_backward(C.byref(s), x, lengths, weight, bias, initial, d, dlast, gx, gw, gb, gi, ws, None)


def size_of(fn, *args):
    n = C.c_size_t()
    assert fn(*args, C.byref(n)) == OK
    return n.value


@pytest.mark.parametrize("bad", [dict(B=0), dict(T=0), dict(C_=0), dict(K=1), dict(K=9), dict(act=2), dict(dtype=3), dict(dtype=-1), dict(T=(1 << 30) + 1),
                                 dict(C_=(1 << 24) + 1), dict(B=1 << 30, T=1 << 20)])
def test_convolution_shapes_that_are_refused(lib, bad):
    s, n = conv(**bad), C.c_size_t()
    assert lib.esrnn_convolution_workspace_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert conv_forward(lib, s) == CONFIG and conv_backward(lib, s) == CONFIG


def test_convolution_arguments_that_are_refused(lib):
    ok = conv()
    assert 0 < size_of(lib.esrnn_convolution_workspace_bytes, C.byref(ok)) < 1 << 20
    assert lib.esrnn_convolution_workspace_bytes(None, C.byref(C.c_size_t())) == NULL
    for name in ("x", "weight", "out"):
        assert conv_forward(lib, ok, **{name: None}) == NULL
    for name in ("x", "weight", "d", "gx", "gw", "ws"):
        assert conv_backward(lib, ok, **{name: None}) == NULL
    for name in ("x", "weight", "bias", "initial", "out", "last", "lengths"):
        assert conv_forward(lib, ok, **{name: odd(P[13])}) == CONFIG, name
    for name in ("x", "weight", "bias", "initial", "d", "dlast", "gx", "gw", "gb", "gi"):
        assert conv_backward(lib, ok, **{name: odd(P[13], 2)}) == CONFIG, name
    assert conv_backward(lib, ok, ws=odd(P[12], 64)) == WORKSPACE
    for stride in ((0, 64), (64, 64), (30 * 64, 63), (-1, 64), (1 << 41, 64)):
        assert conv_forward(lib, conv(out_stride=stride)) == CONFIG and conv_backward(lib, conv(grad_x_stride=stride)) == CONFIG
    assert conv_forward(lib, conv(x_stride=(-64, 64))) == CONFIG and conv_backward(lib, conv(grad_out_stride=(64, 1 << 40))) == CONFIG
    # arrays that are written over others
    assert conv_forward(lib, ok, out=P[0]) == CONFIG and conv_forward(lib, ok, out=odd(P[0], 64 * 4)) == CONFIG
    assert conv_forward(lib, ok, last=P[3]) == CONFIG and conv_forward(lib, ok, last=odd(P[3], 16)) == CONFIG and conv_forward(lib, ok, out=P[3]) == CONFIG
    assert conv_backward(lib, ok, gx=P[0]) == CONFIG and conv_backward(lib, ok, gx=P[6]) == CONFIG and conv_backward(lib, ok, gi=P[7]) == CONFIG
    assert conv_backward(lib, ok, gw=P[1]) == CONFIG and conv_backward(lib, ok, gb=P[9]) == CONFIG and conv_backward(lib, ok, gb=P[2]) == CONFIG
    # halves of one array are no overlap, halves that reach into each other are
    halves = conv(x_stride=(30 * 128, 128), out_stride=(30 * 128, 128))
    assert conv_forward(lib, halves, out=odd(P[0], 4 * 63)) == CONFIG


def test_convolution_steps_that_are_refused(lib):
    def step(rows=2, pool=4, C_=8, K=4, act=1, dtype=0, x=P[0], w=P[1], b=P[2], slots=P[3], state=P[4], out=P[5], xs=8, os_=8):
        s = ss.ConvolutionStepShape(rows, pool, C_, K, act, dtype, xs, os_)
        return lib.esrnn_convolution_step(C.byref(s), x, w, b, slots, state, out, None)
    assert step(rows=0) == OK and step(rows=0, x=None, w=None, state=None, out=None) == OK
    for bad in (dict(K=1), dict(K=9), dict(act=2), dict(dtype=5), dict(rows=-1), dict(C_=0), dict(pool=-1), dict(slots=None, rows=5), dict(xs=-8), dict(os_=7),
                dict(xs=1 << 41), dict(state=odd(P[4], 2)), dict(out=P[0]), dict(state=P[5]), dict(slots=odd(P[3]))):
        assert step(**bad) == CONFIG, bad
    for name in ("x", "w", "state", "out"):
        assert step(**{name: None}) == NULL
    assert lib.esrnn_convolution_step(None, P[0], P[1], None, None, P[4], P[5], None) == NULL


# ---- selective scan ----
def select(B=2, T=30, C_=64, N=16, G=1, kind=0, dtype=0, **strides):
    s = ss.SelectiveShape()
    s.B, s.T, s.C, s.N, s.G, s.delta_kind, s.dtype = B, T, C_, N, G, kind, dtype
    for name in ("x", "delta", "out", "grad_out", "grad_x", "grad_delta"):
        getattr(s, name + "_stride")[0], getattr(s, name + "_stride")[1] = strides.get(name, (T * C_, C_))
    for name in ("b", "c", "grad_b", "grad_c"):
        getattr(s, name + "_stride")[0], getattr(s, name + "_stride")[1] = strides.get(name, (T * G * N, G * N))
    return s


def select_forward(lib, s, x=P[0], delta=P[1], A=P[2], b=P[3], c=P[4], D=P[5], bias=P[6], lengths=None, initial=P[7], out=P[8], last=P[9], saved=P[10], ws=P[11]):
    return lib.esrnn_selective_forward(C.byref(s), x, delta, A, b, c, D, bias, lengths, initial, out, last, saved, ws, None)


def select_backward(lib, s, x=P[0], delta=P[1], A=P[2], b=P[3], c=P[4], D=P[5], bias=P[6], lengths=None, saved=P[7], d=P[8], dlast=P[9], ws=P[10], **grads):
    at = dict(x=P[11], delta=P[12], b=P[13], c=P[14], A=P[15], D=odd(P[15], 1 << 30), bias=odd(P[15], 1 << 31), initial=odd(P[15], 1 << 32)) | grads
    g = ss.SelectiveGrads(**{k: v.value if v else None for k, v in at.items()})
    return lib.esrnn_selective_backward(C.byref(s), x, delta, A, b, c, D, bias, lengths, saved, d, dlast, C.byref(g), ws, None)


@pytest.mark.parametrize("bad", [dict(B=0), dict(T=0), dict(C_=0), dict(N=0), dict(N=65), dict(G=0), dict(G=3), dict(G=128), dict(kind=2), dict(dtype=3), dict(T=(1 << 30) + 1),
                                 dict(B=1 << 23, T=1), dict(C_=(1 << 24) + 64), dict(B=1 << 12, T=1 << 30)])
def test_selective_shapes_that_are_refused(lib, bad):
    s, n = select(**bad), C.c_size_t()
    assert lib.esrnn_selective_workspace_bytes(C.byref(s), 0, C.byref(n)) == CONFIG and lib.esrnn_selective_saved_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert select_forward(lib, s) == CONFIG and select_backward(lib, s) == CONFIG


def test_selective_sizes(lib):
    saved = lambda **kw: size_of(lib.esrnn_selective_saved_bytes, C.byref(select(**kw)))  # noqa: E731
    work = lambda reverse, **kw: size_of(lib.esrnn_selective_workspace_bytes, C.byref(select(**kw)), reverse)  # noqa: E731
    # a state of every channel, of whole tiles and fours, for every eight positions
    for T in (1, 8, 9, 1000):
        for C_, N in ((64, 16), (50, 5), (200, 33)):
            padded = {16: 16, 5: 8, 33: 64}[N]
            assert saved(T=T, C_=C_, N=N) == 4 * 2 * -(-T // 8) * -(-C_ // 64) * 64 * padded
    # forward: maps of segments and widened rows; in reverse also a partial gradient of b and c for every tile, which is one array of x's in fp32 at 16 states
    x = 4 * 4 * 4096 * 2048
    kw = dict(B=4, T=4096, C_=2048)
    assert work(0, **kw) < 0.5 * x and 0.5 * x < work(1, **kw) < 1.5 * x
    assert work(0, B=1, T=1, C_=1, N=1) % 256 == 0


def test_selective_arguments_that_are_refused(lib):
    ok = select()
    for name in ("x", "delta", "A", "b", "c", "out", "ws"):
        assert select_forward(lib, ok, **{name: None}) == NULL, name
    for name in ("x", "delta", "A", "b", "c", "saved", "d", "ws"):
        assert select_backward(lib, ok, **{name: None}) == NULL, name
    g = ss.SelectiveGrads()
    assert lib.esrnn_selective_backward(C.byref(ok), *P[:7], None, P[7], P[8], None, None, P[10], None) == NULL
    assert lib.esrnn_selective_backward(C.byref(ok), *P[:7], None, P[7], P[8], None, C.byref(g), P[10], None) == NULL
    for name in ("x", "delta", "A", "b", "c", "D", "bias", "initial", "out", "last", "lengths"):
        assert select_forward(lib, ok, **{name: odd(P[13], 2)}) == CONFIG, name
    for name in ("ws", "saved"):
        assert select_forward(lib, ok, **{name: odd(P[13], 64)}) == WORKSPACE
    for stride in ((0, 64), (64, 64), (30 * 64, 63), (-1, 64)):
        assert select_forward(lib, select(out=stride)) == CONFIG
        assert select_backward(lib, select(grad_x=stride)) == CONFIG and select_backward(lib, select(grad_delta=stride)) == CONFIG
    assert select_backward(lib, select(grad_b=(30 * 16, 15))) == CONFIG and select_backward(lib, select(grad_c=(0, 16))) == CONFIG
    assert select_forward(lib, select(b=(-1, 16))) == CONFIG and select_forward(lib, select(c=(1 << 41, 16))) == CONFIG
    # over each other
    for name in ("x", "delta", "b", "c"):
        assert select_forward(lib, ok, **{name: P[8]}) == CONFIG
    assert select_forward(lib, ok, last=P[7]) == CONFIG and select_forward(lib, ok, last=odd(P[7], 64)) == CONFIG and select_forward(lib, ok, last=P[2]) == CONFIG
    grads = lambda **kw: lib.esrnn_selective_backward(C.byref(ok), *P[:7], None, P[7], P[8], P[9], C.byref(ss.SelectiveGrads(**kw)), P[10], None)  # noqa: E731
    base = dict(x=P[11].value, delta=P[12].value, b=P[13].value, c=P[14].value, A=P[15].value, D=P[15].value + (1 << 30), bias=P[15].value + (1 << 31),
                initial=P[15].value + (1 << 32))
    for name, at in (("x", P[0]), ("delta", P[1]), ("x", P[8]), ("x", P[12]), ("b", P[3]), ("c", P[13]), ("A", P[2]), ("D", P[5]), ("bias", P[6]), ("initial", P[9]),
                     ("D", odd(P[15], 1 << 31)), ("A", odd(P[15], 1 << 30)), ("initial", odd(P[15], 64))):
        assert grads(**(base | {name: at.value})) == CONFIG, name
    # b and c as slices of one projection may not reach into each other when they are written
    one = select(grad_b=(30 * 32, 32), grad_c=(30 * 32, 32))
    g = ss.SelectiveGrads(**(base | {"c": base["b"] + 15 * 4}))
    assert lib.esrnn_selective_backward(C.byref(one), *P[:7], None, P[7], P[8], P[9], C.byref(g), P[10], None) == CONFIG


def test_selective_steps_that_are_refused(lib):
    def step(rows=2, pool=4, C_=8, N=4, G=2, kind=0, dtype=0, x=P[0], delta=P[1], A=P[2], b=P[3], c=P[4], D=P[5], bias=P[6], slots=P[7], state=P[8], out=P[9],
             xs=8, ds=8, bs=8, cs=8, os_=8):
        s = ss.SelectiveStepShape(rows, pool, C_, N, G, kind, dtype, xs, ds, bs, cs, os_)
        return lib.esrnn_selective_step(C.byref(s), x, delta, A, b, c, D, bias, slots, state, out, None)
    assert step(rows=0) == OK and step(rows=0, x=None, state=None, out=None) == OK
    for bad in (dict(N=0), dict(N=65), dict(G=0), dict(G=3), dict(kind=2), dict(dtype=5), dict(rows=-1), dict(C_=0), dict(pool=-1), dict(slots=None, rows=5), dict(xs=-8),
                dict(os_=7), dict(bs=1 << 41), dict(state=odd(P[8], 2)), dict(A=odd(P[2])), dict(out=P[0]), dict(out=P[1]), dict(out=P[3]), dict(out=P[4])):
        assert step(**bad) == CONFIG, bad
    for name in ("x", "delta", "A", "b", "c", "state", "out"):
        assert step(**{name: None}) == NULL


# ---- block norm ----
def block(rows=5, C_=64, gate=1, dtype=0, stream=0, eps=1e-5, **strides):
    s = ss.BlockNormShape()
    s.rows, s.C, s.gate, s.dtype, s.stream_dtype, s.eps = rows, C_, gate, dtype, stream, eps
    for name in ("y", "gate", "residual", "sum", "out", "grad_out", "grad_sum", "grad_y", "grad_gate", "grad_residual"):
        setattr(s, name + "_stride", strides.get(name, C_))
    return s


OPERANDS = dict(y=P[0], gate=P[1], residual=P[2], exists=None, post_weight=P[3], scale=P[4], pre_weight=P[5])
values = lambda d: {k: v.value if v else None for k, v in d.items()}  # noqa: E731


def block_forward(lib, s, sum=P[6], out=P[7], stats=P[8], **operands):
    o = ss.BlockNormOperands(**values(OPERANDS | operands))
    return lib.esrnn_block_norm_forward(C.byref(s), C.byref(o), sum, out, stats, None)


GRADS = dict(y=P[9], gate=P[10], residual=P[11], post_weight=P[12], scale=P[13], pre_weight=P[14])


def block_backward(lib, s, stats=P[8], d=P[6], dsum=P[7], ws=P[15], grads={}, **operands):
    o, g = ss.BlockNormOperands(**values(OPERANDS | operands)), ss.BlockNormGrads(**values(GRADS | grads))
    return lib.esrnn_block_norm_backward(C.byref(s), C.byref(o), stats, d, dsum, C.byref(g), ws, None)


@pytest.mark.parametrize("bad", [dict(rows=0), dict(C_=0), dict(C_=8193), dict(gate=3), dict(gate=-1), dict(dtype=3), dict(dtype=1, stream=2), dict(stream=1), dict(eps=0.0), dict(eps=-1.0),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(rows=(1 << 30) + 1)])
def test_block_norm_shapes_that_are_refused(lib, bad):
    s, n = block(**bad), C.c_size_t()
    assert lib.esrnn_block_norm_workspace_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert block_forward(lib, s) == CONFIG and block_backward(lib, s) == CONFIG


def test_block_norm_arguments_that_are_refused(lib):
    ok = block()
    assert size_of(lib.esrnn_block_norm_workspace_bytes, C.byref(block(rows=1 << 30, C_=8192))) <= 4096 * 3 * 8192 * 4
    # what there has to be, and what must not
    for name in ("y", "gate"):
        assert block_forward(lib, ok, **{name: None}) == NULL
    assert block_forward(lib, ok, sum=None) == NULL and block_forward(lib, ok, out=None) == NULL
    assert block_forward(lib, ok, residual=None) == CONFIG and block_forward(lib, ok, pre_weight=None) == CONFIG and block_forward(lib, block(gate=0)) == CONFIG
    for name in ("y", "gate", "residual", "post_weight", "scale", "pre_weight"):
        assert block_backward(lib, ok, grads={name: None}) == NULL, name
    assert block_backward(lib, ok, d=None) == NULL and block_backward(lib, ok, stats=None) == NULL and block_backward(lib, ok, ws=None) == NULL
    assert block_backward(lib, ok, post_weight=None) == CONFIG and block_backward(lib, ok, scale=None) == CONFIG and block_backward(lib, block(gate=0)) == CONFIG
    assert block_backward(lib, ok, residual=None, grads={"residual": None}) == CONFIG            # a gradient of a sum that there is not
    assert block_backward(lib, ok, pre_weight=None, grads={"pre_weight": None}) == CONFIG       # one of an output that there is not
    assert block_backward(lib, ok, ws=odd(P[15], 64)) == WORKSPACE
    # alignment and strides
    for name in OPERANDS:
        assert block_forward(lib, ok, **{name: odd(P[12], 2)}) == CONFIG, name
    for name in ("y", "gate", "residual"):
        assert block_forward(lib, block(**{name: -64})) == CONFIG and block_forward(lib, block(**{name: 1 << 41})) == CONFIG
    for name in ("sum", "out"):
        assert block_forward(lib, block(**{name: 63})) == CONFIG
    for name in ("grad_y", "grad_gate", "grad_residual"):
        assert block_backward(lib, block(**{name: 63})) == CONFIG
    # over each other
    for at in (P[0], P[1], P[2], P[6]):
        assert block_forward(lib, ok, out=at) == CONFIG
    assert block_forward(lib, ok, sum=P[0]) == CONFIG and block_forward(lib, ok, sum=odd(P[0], 4)) == CONFIG
    assert block_forward(lib, ok, sum=P[2]) == CONFIG                                           # in place, but a reverse pass would need the residual
    assert block_forward(lib, block(sum=128), sum=P[2], stats=None) == CONFIG                   # in place at other strides
    for name in ("y", "gate", "residual"):
        for at in (P[0], P[1], P[2], P[6], P[7]):
            assert block_backward(lib, ok, grads={name: at}) == CONFIG, name
    for name in ("post_weight", "scale", "pre_weight"):
        for at in (P[3], P[4], P[5]):
            assert block_backward(lib, ok, grads={name: at}) == CONFIG, name
    assert block_backward(lib, ok, grads={"scale": GRADS["post_weight"]}) == CONFIG and block_backward(lib, ok, grads={"gate": GRADS["y"]}) == CONFIG


# ---- arrays of different kinds at one place, and sizes that no launch has ----
def test_arrays_at_one_place_are_refused(lib):
    c, s, n = conv(), select(), block()
    for written, read in ((dict(out=P[1]), "weight"), (dict(out=P[2]), "bias"), (dict(last=P[1]), "weight"), (dict(last=P[0]), "x"), (dict(last=P[4]), "out")):
        assert conv_forward(lib, c, **written) == CONFIG, read
    for written in (dict(gx=P[1]), dict(gx=P[7]), dict(gw=P[0]), dict(gw=P[6]), dict(gi=P[3]), dict(gi=P[9]), dict(ws=P[0]), dict(ws=P[8])):
        assert conv_backward(lib, c, **written) == CONFIG, written
    for written in (dict(out=P[2]), dict(last=P[0]), dict(last=P[8]), dict(saved=P[0]), dict(saved=P[7]), dict(saved=P[11]), dict(ws=P[2]), dict(ws=P[8])):
        assert select_forward(lib, s, **written) == CONFIG, written
    for at in (P[7], P[8], P[11]):
        assert select_backward(lib, s, ws=at) == CONFIG
    places = dict(x=P[11], delta=P[12], b=P[13], c=P[14], A=P[15], D=odd(P[15], 1 << 30), bias=odd(P[15], 1 << 31), initial=odd(P[15], 1 << 32))
    for name, at in (("x", P[7]), ("A", P[9]), ("b", P[2]), ("D", P[6]), ("bias", P[5]), ("initial", P[7]), ("c", P[10]), ("delta", P[4])):
        g = ss.SelectiveGrads(**values(places | {name: at}))
        assert lib.esrnn_selective_backward(C.byref(s), *P[:7], None, P[7], P[8], P[9], C.byref(g), P[10], None) == CONFIG, name
    for written in (dict(stats=P[0]), dict(stats=P[2]), dict(stats=P[5]), dict(stats=P[7]), dict(out=P[3]), dict(sum=P[4])):
        assert block_forward(lib, n, **written) == CONFIG, written
    for at in (P[0], P[3], P[6], P[7], P[8], P[9], P[12]):
        assert block_backward(lib, n, ws=at) == CONFIG
    assert block_backward(lib, n, grads={"y": P[8]}) == CONFIG and block_backward(lib, n, grads={"scale": P[6]}) == CONFIG
    step = ss.SelectiveStepShape(2, 4, 8, 4, 2, 0, 0, 8, 8, 8, 8, 8)
    for state in (*P[:8], P[9]):
        assert lib.esrnn_selective_step(C.byref(step), *P[:8], state, P[9], None) == CONFIG
    for out in P[:8]:
        assert lib.esrnn_selective_step(C.byref(step), *P[:8], P[8], out, None) == CONFIG
    step = ss.ConvolutionStepShape(2, 4, 8, 4, 1, 0, 8, 8)
    for state, out in ((P[0], P[5]), (P[1], P[5]), (P[2], P[5]), (P[3], P[5]), (P[4], P[4]), (P[4], P[0]), (P[4], P[1]), (P[4], P[2]), (P[4], P[3])):
        assert lib.esrnn_convolution_step(C.byref(step), *P[:4], state, out, None) == CONFIG


def test_launches_have_fewer_than_2_to_the_32_threads(lib):
    n = C.c_size_t()
    for most, more in ((dict(B=(1 << 24) - 1, T=3, C_=5), dict(B=1 << 24, T=3, C_=5)), (dict(B=1, T=128, C_=1 << 24), dict(B=64, T=129, C_=1 << 24)),
                       (dict(B=1 << 23, T=1, C_=64), dict(B=1 << 23, T=1, C_=65))):
        assert lib.esrnn_convolution_workspace_bytes(C.byref(conv(**most)), C.byref(n)) == OK
        assert lib.esrnn_convolution_workspace_bytes(C.byref(conv(**more)), C.byref(n)) == CONFIG and conv_forward(lib, conv(**more)) == CONFIG
    for most, more in ((dict(B=1 << 20, T=1, C_=64), dict(B=(1 << 20) + 1, T=1, C_=64)), (dict(B=1, T=1, C_=64 << 15), dict(B=1, T=1, C_=(64 << 15) + 64)),
                       (dict(B=1, T=1, C_=1 << 15, G=1 << 15), dict(B=1, T=1, C_=1 << 16, G=1 << 16))):
        assert lib.esrnn_selective_workspace_bytes(C.byref(select(**most)), 1, C.byref(n)) == OK
        assert lib.esrnn_selective_workspace_bytes(C.byref(select(**more)), 1, C.byref(n)) == CONFIG and select_forward(lib, select(**more)) == CONFIG


def test_null_shapes(lib):
    n = C.c_size_t()
    assert lib.esrnn_selective_workspace_bytes(None, 0, C.byref(n)) == NULL and lib.esrnn_selective_saved_bytes(C.byref(select()), None) == NULL
    assert lib.esrnn_block_norm_workspace_bytes(None, C.byref(n)) == NULL and lib.esrnn_block_norm_forward(None, None, None, None, None, None) == NULL
    assert conv_forward(lib, None) == NULL
