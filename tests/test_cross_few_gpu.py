"""Cross attention of few queries a key head, which has a kernel of its own, against its formulas in 64 bits (tolerances: tests/test_cross_gpu.py).

Sizes on either side of what that kernel divides: 8 query rows of a key head, batches of 16 keys, 4 warps, up to 8 parts of the keys."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig
from test_cross_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [1, 15, 16, 17, 63, 64, 65, 127, 511, 512, 513, 1000])
@pytest.mark.parametrize("heads", [(1, 1, 64), (4, 2, 128), (8, 1, 128), (9, 1, 64)])
def test_key_counts(K, heads):
    H, G, d = heads
    Case(2, 1, K, H, G, d).check(backward=False)


@pytest.mark.parametrize("d", [8, 16, 24, 56, 64, 72, 104, 128])
@pytest.mark.parametrize("order", ["heads_first", "tokens_first", "wide"])
def test_head_dims_and_strides(d, order):
    Case(3, 2, 90, 6, 2, d, order).check(backward=False)


@pytest.mark.parametrize("rows", [(1, 2), (1, 3), (2, 4), (3, 2), (7, 1), (8, 1), (2, 3), (1, 5)])
@pytest.mark.parametrize("keys", ["lengths", "mask", "both"])
def test_rows_and_keys_that_do_not_count(rows, keys):
    """Tokens and heads of a key head in the eight rows; samples without keys, with negative and with too large lengths."""
    N, group = rows
    Case(6, N, 333, 2 * group, 2, 64, "wide", keys).check(backward=False)


@pytest.mark.parametrize("shape", [(1, 1, 20000, 8, 8, 128), (200, 1, 130, 2, 2, 64), (700, 2, 40, 1, 1, 128), (5, 1, 3001, 32, 8, 80)])
def test_parts_and_many_heads(shape):
    Case(*shape, keys="lengths").check(backward=False)


def test_scores_from_low_to_high():
    """Maxima that grow from key to key, so that what was summed is weighed again at every step."""
    c = Case(1, 1, 900, 4, 4, 64, scale=0.5)
    c.q.abs_()
    c.k.copy_((torch.arange(900, device="cuda") / 300.0)[:, None].expand(900, 64).to(torch.bfloat16))
    c.check(backward=False)


def test_padded_batch_captured():
    """A captured call takes the lengths of its replay."""
    c = Case(4, 1, 257, 8, 2, 128, keys="lengths", spoil=False)
    out = torch.empty_like(c.q)
    c.attention.forward(c.q, c.k, c.v, out, None, c.lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attention.forward(c.q, c.k, c.v, out, None, c.lengths)
    for values in ([257, 0, 64, 1], [0, 0, 0, 0], [16, 255, 257, 128]):
        c.lengths.copy_(torch.tensor(values, dtype=torch.int32))
        out.fill_(float("nan"))
        graph.replay()
        want = torch.empty_like(out)
        B.CrossAttention(CrossAttentionConfig(128, 8, 2, c.scale)).forward(c.q, c.k, c.v, want, None, c.lengths)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all((out[b] == 0).all() for b, n in enumerate(values) if n == 0)
