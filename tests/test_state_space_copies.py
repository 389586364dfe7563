"""What the reverse pass of the selective scan copies of b and c where it cannot read them as they are: what something reads, and no more."""
import ctypes as C

import pytest

from paper_1907_03329_amd import state_space as ss
from tests.test_state_space_host import lib, select, size_of  # noqa: F401  (a fixture)


@pytest.mark.parametrize("B,T,C_,N,G", [(100, 8, 64, 16, 1), (37, 1, 130, 5, 2), (1, 4096, 64, 16, 1), (3, 2000, 300, 7, 3), (4, 1024, 256, 32, 1), (1, 8192, 64, 64, 1)])
def test_rows_in_the_workspace(lib, B, T, C_, N, G):  # noqa: F811
    """fp32 rows of c for the maps of segments, and none where there is one segment.  Beside them: b and c by pieces of eight positions, a share of both gradients
    for every tile, and for each segment its maps and its sums for A, D and bias."""
    states, slices = 4 if N <= 4 else 8 if N <= 8 else 16, 1 if N <= 16 else 2 if N <= 32 else 4
    tiles, one = -(-(C_ // G) // 64), G * states * slices
    pieces = B * -(-T // 8) * 8 * one
    work = size_of(lib.esrnn_selective_workspace_bytes, C.byref(select(B=B, T=T, C_=C_, N=N, G=G)), 1) // 4
    rest = work - 2 * pieces - 2 * pieces * tiles
    lines = B * G * tiles * slices * 64
    single = lines * (states + 2)
    if T <= 8:
        assert single <= rest < single + 256
    else:
        assert any(0 <= rest - B * T * one - segments * lines * (2 * states + 3) < 256 for segments in range(2, -(-T // 8) + 1))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N", [("float16", 16), ("float32", 7), ("bfloat16", 20)])
def test_launches_of_one_segment(dtype, N):
    """b and c by pieces, the gradients, and the sums."""
    import torch
    dt, B, T, C_ = getattr(torch, dtype), 3, 8, 64
    wide, narrow = (lambda: torch.randn(B, T, C_, device="cuda").to(dt)), (lambda: torch.randn(B, T, 1, N, device="cuda").to(dt))
    x, delta, d, b, c = wide(), wide(), wide(), narrow(), narrow()
    A = -torch.rand(C_, N, device="cuda")
    layer = ss.SelectiveScan(B, T, C_, N, dtype=dt)
    layer.forward(x, delta, A, b, c)
    eager = [t.clone() for t in layer.backward(x, delta, A, b, c, d)]
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        grads = layer.backward(x, delta, A, b, c, d)
    nodes = C.c_size_t()
    runtime = ss._library()     # (which is linked to it)
    assert runtime.hipGraphGetNodes(C.c_void_p(graph.raw_cuda_graph()), None, C.byref(nodes)) == 0
    assert nodes.value == 3
    for _ in range(3):
        for t in grads:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(grads, eager))
