"""Outputs over inputs in other places than the input's own rows are refused before anything runs."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig, LayerNormConfig

pytestmark = pytest.mark.gpu


def refused(call, *args):
    with pytest.raises(B.FFError) as e:
        call(*args)
    assert e.value.status == 1 and "over" in str(e.value)


def test_layer_norm():
    norm = B.LayerNorm(LayerNormConfig(64))
    buffer = torch.randn(4096, device="cuda").to(torch.bfloat16)
    x, other = buffer.as_strided((2, 10, 64), (640, 64, 1)), buffer.as_strided((2, 10, 64), (1280, 128, 1))
    w, dw, db = (torch.randn(64, device="cuda") for _ in range(3))
    dy, before = torch.randn(2, 10, 64, device="cuda").to(torch.bfloat16), buffer.clone()
    refused(norm.forward, x, w, None, other)
    refused(norm.backward, x, w, dy, other, dw, db)
    refused(norm.backward, dy, w, x, other, dw, db)
    refused(norm.backward, x, w, dy, torch.empty_like(dy), dw, dw)
    refused(norm.backward, x, w, dy, torch.empty_like(dy), w, db)
    refused(norm.backward, x, w, dy, torch.empty_like(dy), dw, w)
    assert torch.equal(buffer, before)
    want = torch.empty_like(dy)
    norm.forward(x, w, None, want)
    norm.forward(x, w, None, x)
    assert torch.equal(x, want)


@pytest.mark.parametrize("queries", [1, 40])
def test_cross_attention(queries):
    attention = B.CrossAttention(CrossAttentionConfig(64, 4, 4))
    buffer = torch.randn(1 << 16, device="cuda").to(torch.bfloat16)
    q = buffer.as_strided((2, 4, queries, 64), (256 * queries, 64, 256, 1))
    other = buffer.as_strided((2, 4, queries, 64), (256 * queries, 64 * queries, 64, 1) if queries > 1 else (512, 128, 64, 1))
    k, v = (torch.randn(2, 4, queries, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    before = buffer.clone()
    refused(attention.forward, q, k, v, other)
    refused(attention.forward, q, k, v, k)
    refused(attention.forward, q, k, v, v)
    assert torch.equal(buffer, before)
    want = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    attention.forward(q, k, v, want)
    attention.forward(q, k, v, q)
    assert torch.equal(q, want)
