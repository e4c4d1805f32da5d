"""Which kernel a cross attention call launches, read from a captured graph: the few-rows kernel serves at most eight query rows of a key head, and of
those the sizes that tests/test_cross_few_gpu.py runs; long states of few heads go to the tile kernel, which divides them further."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu
driver = pytest.importorskip("cuda.bindings.driver")


def launched(graph):
    """Names of the kernels in a captured graph."""
    def checked(result):
        assert result[0] == driver.CUresult.CUDA_SUCCESS, result[0]
        return result[1:]
    raw = driver.CUgraph(graph.raw_cuda_graph())
    nodes, count = checked(driver.cuGraphGetNodes(raw, checked(driver.cuGraphGetNodes(raw))[1]))
    found = set()
    for node in nodes[:count]:
        if checked(driver.cuGraphNodeGetType(node))[0] == driver.CUgraphNodeType.CU_GRAPH_NODE_TYPE_KERNEL:
            p = checked(driver.cuGraphKernelNodeGetParams(node))[0]
            name = checked(driver.cuFuncGetName(p.func) if int(p.func) else driver.cuKernelGetName(p.kern))[0].decode()
            found |= {k for k in ("cross_few_kernel", "cross_forward_kernel", "cross_join_kernel") if k in name}
    return found


def kernels(batch, N, K, H, G, d, lengths=False):
    q = torch.zeros(batch, H, N, d, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(batch, G, K, d, dtype=torch.bfloat16, device="cuda")
    n = torch.full((batch,), K, dtype=torch.int32, device="cuda") if lengths else None
    a, out = B.CrossAttention(CrossAttentionConfig(d, H, G)), torch.empty_like(q)
    a.forward(q, k, k, out, lengths=n)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        a.forward(q, k, k, out, lengths=n)
    return launched(graph)


@pytest.mark.parametrize("shape", [(2, 1, K, H, G, d) for K in (1, 64, 513, 1000) for H, G, d in ((1, 1, 64), (4, 2, 128), (8, 1, 128))] +
                         [(3, 2, 90, 6, 2, 56), (6, 3, 333, 4, 2, 64), (6, 1, 333, 10, 2, 64), (1, 1, 20000, 8, 8, 128), (200, 1, 130, 2, 2, 64),
                          (700, 2, 40, 1, 1, 128), (5, 1, 3001, 32, 8, 80), (1, 1, 900, 4, 4, 64), (4, 1, 257, 8, 2, 128)])
def test_few_rows(shape):
    for lengths in (False, True):
        assert kernels(*shape, lengths) == {"cross_few_kernel"}


@pytest.mark.parametrize("shape", [(2, 1, 1000, 9, 1, 64), (2, 9, 300, 1, 1, 64), (2, 3, 200, 12, 4, 128), (1, 300, 200, 2, 2, 64)])
def test_more_rows(shape):
    assert "cross_few_kernel" not in kernels(*shape)


def test_either_side_of_the_choice():
    """One head of 64: 16,000 states by the few-rows kernel, 32,000 by tiles."""
    assert kernels(1, 1, 16000, 1, 1, 64) == {"cross_few_kernel"}
    assert kernels(1, 1, 32000, 1, 1, 64) == {"cross_forward_kernel", "cross_join_kernel"}


@pytest.mark.parametrize("shape", [(1, 1, 32000, 1, 1, 64), (1, 2, 33333, 4, 1, 128), (2, 8, 40001, 1, 1, 80)])
@pytest.mark.parametrize("keys", ["all", "lengths"])
def test_few_rows_by_tiles(shape, keys):
    """What the tile kernel makes of few rows against long states, against the formulas."""
    assert "cross_few_kernel" not in kernels(*shape, keys == "lengths")
    Case(*shape, keys=keys).check(backward=False)
