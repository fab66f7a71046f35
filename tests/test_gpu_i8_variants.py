"""Every kernel, tile and split that the integer product's choice has, each on a whole result.

The bar is that of test_gpu_i8.py: the sum is exact, then three FP32 roundings and one to bf16.
"""
import ctypes
import re

import pytest
import torch

from test_gpu_i8 import b, check_product, codes_of  # noqa: F401

pytestmark = pytest.mark.gpu


class _KernelNode(ctypes.Structure):
    """CUDA_KERNEL_NODE_PARAMS_v2"""
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3), ("smem", ctypes.c_uint), ("params", ctypes.c_void_p),
                ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def product_kernel(call):
    """What a captured call launches of the product's kernels: ("pair" or "split", tokens of a tile, stages of the ring or None, CTAs that share a tile's K,
    CTAs of the grid)."""
    cu = ctypes.CDLL("libcuda.so.1")
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    raw, n = ctypes.c_void_p(int(graph.raw_cuda_graph())), ctypes.c_size_t(0)
    assert cu.cuGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert cu.cuGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    found = []
    for node in nodes:
        p, name, cluster = _KernelNode(), ctypes.c_char_p(), (ctypes.c_uint * 16)()
        if cu.cuGraphKernelNodeGetParams_v2(ctypes.c_void_p(node), ctypes.byref(p)) != 0:
            continue
        assert (cu.cuFuncGetName(ctypes.byref(name), ctypes.c_void_p(p.func)) if p.func else cu.cuKernelGetName(ctypes.byref(name), ctypes.c_void_p(p.kern))) == 0
        m = re.search(r"i8_(split|pair)_kernelILi(\d+)E(?:Li(\d+)E)?", name.value.decode())
        if m:
            assert cu.cuGraphKernelNodeGetAttribute(ctypes.c_void_p(node), 4, cluster) == 0         # the cluster's dimension
            found.append((m[1], int(m[2]), int(m[3]) if m[3] else None, max(cluster[0], 1), p.grid[0]))
    assert len(found) == 1, found
    return found[0]


@pytest.mark.parametrize("M,N,K,kernel", [
    # pairs of CTAs: one tile each, fewer tiles than pairs, a ring that wraps; several tiles each.  (kernel, tokens of a tile, tiles a pair: 1, 2, 3 for more)
    (199, 3971, 4912, ("pair", 64, 1)), (159, 6563, 1072, ("pair", 96, 1)), (225, 7933, 1200, ("pair", 128, 1)), (719, 3401, 496, ("pair", 160, 1)),
    (503, 5609, 912, ("pair", 192, 1)), (619, 5807, 880, ("pair", 224, 1)), (489, 6363, 1632, ("pair", 256, 1)), (125, 19885, 288, ("pair", 64, 3)),
    (89, 20849, 304, ("pair", 96, 2)), (267, 15417, 336, ("pair", 96, 3)), (199, 15055, 480, ("pair", 128, 2)), (197, 20651, 304, ("pair", 128, 3)),
    (301, 15835, 320, ("pair", 160, 2)), (305, 20347, 288, ("pair", 160, 3)), (327, 14499, 1472, ("pair", 192, 2)), (539, 17423, 432, ("pair", 192, 3)),
    (421, 15877, 2064, ("pair", 224, 2)), (661, 16771, 1072, ("pair", 224, 3)), (761, 11931, 2080, ("pair", 256, 2)),
    # one CTA on a tile, or a cluster on its K, with the long ring.  (kernel, tokens of a tile, stages, CTAs of a tile)
    (1, 69, 272, ("split", 16, 12, 1)), (1, 2897, 4448, ("split", 16, 12, 2)), (5, 1615, 2464, ("split", 16, 12, 4)), (9, 73, 1984, ("split", 16, 12, 8)),
    (17, 65, 272, ("split", 32, 11, 1)), (19, 3033, 4976, ("split", 32, 11, 2)), (17, 1607, 3472, ("split", 32, 11, 4)), (18, 65, 2752, ("split", 32, 11, 8)),
    (34, 69, 288, ("split", 64, 9, 1)), (70, 2669, 4464, ("split", 64, 9, 2)), (39, 1893, 2976, ("split", 64, 9, 4)), (40, 67, 2464, ("split", 64, 9, 8)),
    # more tiles than SMs: the short ring
    (13, 20679, 2064, ("split", 16, 6, 1)), (20, 19023, 2064, ("split", 32, 5, 1)), (39, 20567, 1040, ("split", 64, 4, 1)),
])
def test_gemm_i8_every_variant(b, M, N, K, kernel):
    """The whole result by each kernel, tile and split that the choice has, at odd sizes, twice; the captured launch tells which one ran."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("the choice goes by the number of SMs")
    x, w = codes_of(M, K, 1).cuda(), codes_of(N, K, 2).cuda()
    sx, sw = torch.ones(M).cuda(), torch.ones(N).cuda()
    y = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    kind, tokens, stages, ctas, grid = product_kernel(lambda: b.razer_gemm_i8(x, sx, w, sw, y))
    if kind == "pair":
        tiles = -(-N // 256) * -(-M // tokens)
        assert (kind, tokens, min(-(-tiles // (grid // 2)), 3)) == kernel and ctas == 2
    else:
        assert (kind, tokens, stages, ctas) == kernel
    check_product(b, M, N, K, seed=M + N + K)
