"""A video transformer's layer of all parts captured into a graph, forward and the gradients of its second half, and replayed with other inputs,
lengths and modulation: the same bits as the calls one by one."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import configs as C
from paper_2604_22808_b200 import inputs
from paper_2604_22808_b200.configs import CrossAttentionConfig, FFNConfig, LayerNormConfig, RotaryConfig

pytestmark = pytest.mark.gpu


def test_captured_layer():
    cfg = C.R64K.scaled("layer", T=4, H=16, W=16, low_cut=(2, 4, 4), mid_cut=(3, 12, 12), heads=4, b=32, s=2, R=32, m=4)
    H, d, N, D, K, G = cfg.heads, cfg.head_dim, cfg.N, cfg.heads * cfg.head_dim, 77, 2
    gen = torch.Generator("cuda").manual_seed(7)

    def normal(*shape, s=1.0, t=torch.bfloat16):
        return (s * torch.randn(*shape, generator=gen, device="cuda")).to(t)
    Wqkv, Wo, Wq = normal(3, D, D, s=D ** -0.5), normal(D, D, s=D ** -0.5), normal(D, D, s=D ** -0.5)
    Wg, Wu, Wd = normal(D, 2 * D, s=D ** -0.5), normal(D, 2 * D, s=D ** -0.5), normal(2 * D, D, s=(2 * D) ** -0.5)
    x, states, dy = normal(1, N, D), normal(1, K, 2 * G * d), normal(1, N, D)
    mod = [normal(1, D, s=0.2, t=torch.float32) for _ in range(4)]
    lengths = torch.tensor([61], dtype=torch.int32, device="cuda")
    alloc = torch.tensor([1, 2, 4, 7], dtype=torch.uint8, device="cuda")
    norm = B.LayerNorm(LayerNormConfig(D, unit_offset=True))
    plan = B.Plan(cfg, inputs.router_weights(cfg), host_staging=True)
    rotary = B.Rotary(RotaryConfig(d, d, axis_pairs=(16, 24, 24), grid=cfg.grid))
    cross = B.CrossAttention(CrossAttentionConfig(d, H, G))
    ffn = B.GatedFFN(FFNConfig(D, 2 * D))

    def heads(t, n):
        return t.view(1, -1, n, d).transpose(1, 2)
    h, att, h1, out, y, gate, up = (torch.empty(1, N, n, dtype=torch.bfloat16, device="cuda") for n in (D, D, D, D, D, 2 * D, 2 * D))
    lse = torch.empty(1, H, N, device="cuda")
    dx2, dx1, dq, dscale, dshift = (torch.empty_like(t) for t in (x, x, x, mod[0], mod[0]))
    dstates = torch.empty_like(states)
    dWg, dWu, dWd = (torch.empty_like(t) for t in (Wg, Wu, Wd))

    def layer():
        norm.forward(x, mod[0], mod[1], h)
        plan.forward_projected(h, Wqkv, Wo, att, alloc=alloc, timesteps=[500.0], rotary=rotary, eps=1e-6)
        x1 = x + att
        norm.forward(x1, mod[2], mod[3], h1)
        q, k, v = heads(h1 @ Wq, H), heads(states[..., :G * d], G), heads(states[..., G * d:], G)
        cross.forward(q, k, v, heads(out, H), lse, lengths=lengths)
        x2 = x1 + out
        ffn.forward(x2, Wg, Wu, Wd, y, gate, up)
        ffn.backward(x2, Wg, Wu, Wd, gate, up, dy, dx2, dWg, dWu, dWd)
        cross.backward(q, k, v, heads(out, H), lse, heads(dx2, H), heads(dq, H), heads(dstates[..., :G * d], G), heads(dstates[..., G * d:], G), lengths=lengths)
        norm.backward(x1, mod[2], dq @ Wq.t(), dx1, dscale, dshift)
    results = [h, att, h1, out, lse, y, gate, up, dx2, dWg, dWu, dWd, dq, dstates, dx1, dscale, dshift]
    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for n in (61, 77, 0, 5):
        for t in (x, states, dy, *mod):
            t.copy_(normal(*t.shape, s=0.2 if t.dim() == 2 else 1.0, t=t.dtype))
        lengths.fill_(n)
        layer()
        torch.cuda.synchronize()
        want = [t.clone() for t in results]
        for t in results:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))
        assert all(t.isfinite().all() for t in results if t is not lse)
        assert (lse == float("-inf")).all() if n == 0 else lse.isfinite().all()
    assert plan.device_status() == 0 and cross.device_status() == 0 and ffn.device_status() == 0
