"""Arrays of the gated recurrence that overlap are refused before anything is launched (addresses that are looked at, never followed)."""
import ctypes as C

import pytest

from tests.test_layers_host import CONFIG, WS, lib, recurrence  # noqa: F401  (lib: a fixture)


def at(offset):
    """Far apart from the other arrays of a call, but for those at offsets near by."""
    return C.c_void_p((1 << 30) + offset)


APART = [C.c_void_p((1 << 32) * (i + 1)) for i in range(8)]


@pytest.mark.parametrize("first,second", [(0, 0), (0, 4), (4, 0), (0, 4 * (2 * 300 * 64 - 1)), (4 * 64 * 300, 0), (4 * 63, 4 * 300 * 64)])
def test_rows(lib, first, second):  # noqa: F811
    s = recurrence()        # 2 x 300 x 64 fp32, rows one behind the other
    x, gate, out, d, gx, gg, saved = APART[:7]
    forward = lambda x, gate, out: lib.esrnn_recurrence_forward(C.byref(s), x, gate, None, None, out, None, None, WS, None)  # noqa: E731
    assert forward(at(first), gate, at(second)) == CONFIG and forward(x, at(first), at(second)) == CONFIG
    backward = lambda x, gate, d, gx, gg: lib.esrnn_recurrence_backward(C.byref(s), x, gate, None, saved, d, None, gx, gg, None, WS, None)  # noqa: E731
    for i in range(5):
        for j in range(5):
            if i != j and max(i, j) >= 3:
                given = [x, gate, d, gx, gg]
                given[i], given[j] = at(first), at(second)
                assert backward(*given) == CONFIG, (i, j)


def test_states(lib):  # noqa: F811
    s = recurrence()        # states of 2 x 64 floats
    x, gate, out, d, gx, gg, saved = APART[:7]
    near, n = at(4 * 127), 4 * 128
    forward = lambda initial, last, saved: lib.esrnn_recurrence_forward(C.byref(s), x, gate, None, initial, out, last, saved, WS, None)  # noqa: E731
    assert forward(at(0), at(0), None) == CONFIG and forward(at(0), near, None) == CONFIG and forward(near, at(0), None) == CONFIG
    assert forward(at(n), None, at(0)) == CONFIG and forward(None, at(n), at(0)) == CONFIG        # (saved: states of several blocks)
    backward = lambda grad_last, grad_initial, saved: lib.esrnn_recurrence_backward(C.byref(s), x, gate, None, saved, d, grad_last, gx, gg, grad_initial,  # noqa: E731
                                                                                    WS, None)
    assert backward(at(0), at(0), saved) == CONFIG and backward(near, at(0), saved) == CONFIG and backward(None, at(n), at(0)) == CONFIG
