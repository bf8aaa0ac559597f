"""Launches between the blocks as a captured graph has them: every block has work."""
import re

import pytest
import torch

from paper_2106_06998_b200 import binding as xb

pytestmark = pytest.mark.gpu


def blocks_of(call):
    """The kernels that a call launches: their (mangled) names, blocks and threads of a block."""
    driver = pytest.importorskip("cuda.bindings.driver")
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        kept = call()
    ok = driver.CUresult.CUDA_SUCCESS
    handle = driver.CUgraph(graph.raw_cuda_graph())
    status, _, count = driver.cuGraphGetNodes(handle, 0)
    assert status == ok
    status, nodes, count = driver.cuGraphGetNodes(handle, count)
    assert status == ok
    grids = []
    for node in nodes[:count]:
        status, kind = driver.cuGraphNodeGetType(node)
        assert status == ok
        if kind != driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            continue
        status, params = driver.cuGraphKernelNodeGetParams(node)
        assert status == ok
        status, name = driver.cuFuncGetName(params.func)
        assert status == ok
        grids.append((name.decode(), params.gridDimX * params.gridDimY * params.gridDimZ, params.blockDimX))
    del kept
    return grids


@pytest.mark.parametrize("rows,C,group,q", [(8192, 4096, 0, torch.int8), (8192, 4096, 128, torch.float8_e4m3fn), (50000, 72, 0, torch.float8_e4m3fn), (131072, 64, 0, torch.int8)])
def test_values_back_from_8_bits(rows, C, group, q):
    """A thread takes as many octets (of eight values) as the kernel's last template argument says, as far apart as its block is wide: no block begins behind the last octet."""
    Q = torch.ones(rows, C, dtype=torch.int8, device="cuda").view(q)
    scales = torch.ones(rows, -(-C // group) if group else 1, device="cuda")
    (name, blocks, threads), = blocks_of(lambda: xb.xconv_dequantize(Q, scales, group=group))
    each, octets = int(re.search(r"dequantize_kernelI.*Li(\d+)EEEv", name)[1]), rows * (C // 8)
    assert (blocks - 1) * each * threads < octets <= blocks * each * threads
