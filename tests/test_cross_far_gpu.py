"""Cross attention of rows that lie far apart: offsets beyond 2^31 elements along the batch, the heads and the tokens, in every kernel of the forward and
the backward pass.  The same bits as for the same values side by side."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig

pytestmark = pytest.mark.gpu
FAR = (1 << 31) + 128


@pytest.mark.parametrize("axis", ["batch", "head", "token"])
@pytest.mark.parametrize("N,K,d", [(200, 300, 128), (40, 900, 64), (2, 300, 128)])
def test_offsets_beyond_two_to_the_31(axis, N, K, d):
    """Tiles of one head, of several, parts of the keys, and the few-rows kernel.  The tensors share one allocation."""
    B_, H, G = 2, 4, 2
    gen = torch.Generator("cuda").manual_seed(N)
    step = 1 << 20                                           # (between the tensors; none is longer but along `axis`)
    pool = torch.empty(FAR + (1 << 25), dtype=torch.bfloat16, device="cuda")

    def views(heads, tokens, first):
        if axis == "batch":
            st = (FAR, tokens * d, d)
        elif axis == "head":
            st = (tokens * d, FAR // (heads - 1) // 8 * 8 + 8, d)
        else:
            st = (heads * d, d, max(FAR // (tokens - 1) // 8 * 8 + 8, B_ * heads * d))
        return pool.as_strided((B_, heads, tokens, d), (*st, 1), first * step)
    shapes = [(H, N), (G, K), (G, K), (H, N), (H, N), (H, N), (G, K), (G, K)]       # q, k, v, out, dout, dq, dk, dv
    there = [views(*s, i) for i, s in enumerate(shapes)]
    near = [torch.randn(B_, *s, d, generator=gen, device="cuda").to(torch.bfloat16) for s in shapes]
    for i in (0, 1, 2, 4):
        there[i].copy_(near[i])
    lengths = torch.tensor([K, K - 37], dtype=torch.int32, device="cuda")
    a = B.CrossAttention(CrossAttentionConfig(d, H, G))
    for q, k, v, out, dout, dq, dk, dv in (near, there):
        lse = torch.empty(B_, H, N, device="cuda")
        a.forward(q, k, v, out, lse, lengths)
        a.backward(q, k, v, out, lse, dout, dq, dk, dv, lengths)
    assert a.device_status() == 0
    assert all(torch.equal(near[i], there[i]) for i in (3, 5, 6, 7))
