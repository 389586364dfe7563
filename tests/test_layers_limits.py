"""Sizes that a group norm of single positions takes, and those that it refuses (host only)."""
import ctypes as C

import pytest

from tests.test_layers_host import CONFIG, OK, P, WS, lib, norm  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("N,C_,G", [(131072, 4096, 32), ((1 << 23) + 5, 64, 16), (600001, 8192, 2), (1 << 30, 1, 1), (1 << 30, 1024, 1024),
                                    (1 << 20, 1 << 20, 256)])
def test_taken(lib, N, C_, G):  # noqa: F811
    n, s = C.c_size_t(), norm(N, 1, C_, G)
    assert lib.esrnn_group_norm_workspace_bytes(C.byref(s), C.byref(n)) == OK
    assert 0 < n.value <= 2 * 1024 * 2 * 4 * max(C_, 2048)      # rows of sums for some thousand workgroups


@pytest.mark.parametrize("N,T,C_,G", [((1 << 30) + 1, 1, 1, 1), (1 << 30, 1, 1025, 1025), ((1 << 20) + 1, 1, 1 << 20, 256),
                                      (131072, 2, 4096, 32), (131072, 1, 4100, 1)])
def test_refused(lib, N, T, C_, G):  # noqa: F811
    n, s = C.c_size_t(), norm(N, T, C_, G)
    assert lib.esrnn_group_norm_workspace_bytes(C.byref(s), C.byref(n)) == CONFIG
    assert lib.esrnn_group_norm_forward(C.byref(s), P, None, P, P, P, None, WS, None) == CONFIG
