"""Which launches lg_page_fork takes: one for small maps of few sequences, two in which all sequences run at once for
the others. One workgroup works through many short sequences four at a time: 281 us for 512 of 16 slots, 5.8 in two launches."""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _nodes(graph):
    """Nodes of a captured graph."""
    hip = ctypes.CDLL("libamdhip64.so")
    n = ctypes.c_size_t()
    hip.hipGraphGetNodes.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(ctypes.c_size_t)]
    assert hip.hipGraphGetNodes(graph.raw_cuda_graph(), None, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("B,cap,launches", [(1, 256, 1), (4, 256, 1), (8, 512, 1), (8, 2048, 2), (16, 256, 2), (32, 128, 2),
                                            (64, 128, 2), (200, 32, 2), (512, 16, 2)])
def test_launches(B, cap, launches):
    from paper_2604_10044_amd import lg
    i32 = lambda x: torch.as_tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    P = cap // 16
    table, pos = np.arange(B * P).reshape(B, P), np.arange(B * cap).reshape(B, cap)
    t, p, n, ref = i32(table), i32(pos), i32([cap] * B), i32(np.ones(B * P))
    m = lg.page_map(t, p, n, ref, 16)
    ws = torch.empty(lg.lg_page_workspace(m), dtype=torch.uint8, device="cuda")
    parent = i32(np.roll(np.arange(B), 1))
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        lg.lg_page_fork(m, parent, ws)
    assert _nodes(graph) == launches
    for turn in range(1, 4):  # a rotation of the batch
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(t.cpu().numpy(), np.roll(table, turn, 0))
        np.testing.assert_array_equal(p.cpu().numpy(), np.roll(pos, turn, 0))
        assert (ref == 1).all() and (n == cap).all()
