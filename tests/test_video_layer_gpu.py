"""A video transformer's layer of all parts: norm with the sample's scale and shift, the projected attention with rotary positions and
norm of queries and keys, cross attention to padded states, and the feed-forward block; then the gradients of its second half."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import configs as C
from paper_2604_22808_b200 import inputs
from paper_2604_22808_b200.configs import CrossAttentionConfig, FFNConfig, LayerNormConfig, RotaryConfig

pytestmark = pytest.mark.gpu


def norm64(x, w, b, eps, plus):
    c = x - x.mean(-1, keepdim=True)
    n = c * ((c * c).mean(-1, keepdim=True) + eps).rsqrt()
    return n * (plus + w)[:, None] + b[:, None] if w.dim() == 2 else n * (plus + w) + b


def cross64(q, k, v, counts):
    s = (q @ k.transpose(-1, -2)) * q.shape[-1] ** -0.5
    return torch.softmax(s.masked_fill(~counts[:, None, None], float("-inf")), -1) @ v


def close(got, want, steps, what):
    """Within `steps` roundings to bf16 of the tensor's size: what goes through several bf16 tensors on its way."""
    err, size = (got.double() - want).pow(2).mean().sqrt().item(), want.pow(2).mean().sqrt().item()
    assert err <= steps * 2.0 ** -8 * size, f"{what}: {err / size:.3g}"


def test_layer():
    cfg = C.R64K.scaled("layer", T=4, H=16, W=16, low_cut=(2, 4, 4), mid_cut=(3, 12, 12), heads=4, b=32, s=2, R=32, m=4)
    H, d, N, D, K, G = cfg.heads, cfg.head_dim, cfg.N, cfg.heads * cfg.head_dim, 77, 2
    gen = torch.Generator("cuda").manual_seed(5)

    def normal(*shape, s=1.0, t=torch.bfloat16):
        return (s * torch.randn(*shape, generator=gen, device="cuda")).to(t)
    x = normal(1, N, D)
    mod = [normal(1, D, s=0.2, t=torch.float32) for _ in range(4)]                   # scale and shift of two norms
    Wqkv, Wo = normal(3, D, D, s=D ** -0.5), normal(D, D, s=D ** -0.5)
    states, Wq = normal(1, K, 2 * G * d), normal(D, D, s=D ** -0.5)
    lengths = torch.tensor([61], dtype=torch.int32, device="cuda")
    Wg, Wu, Wd = normal(D, 2 * D, s=D ** -0.5), normal(D, 2 * D, s=D ** -0.5), normal(2 * D, D, s=(2 * D) ** -0.5)

    norm = B.LayerNorm(LayerNormConfig(D, unit_offset=True))
    plan = B.Plan(cfg, inputs.router_weights(cfg), host_staging=True)
    rotary = B.Rotary(RotaryConfig(d, d, axis_pairs=(16, 24, 24), grid=cfg.grid))
    cross = B.CrossAttention(CrossAttentionConfig(d, H, G))
    ffn = B.GatedFFN(FFNConfig(D, 2 * D))

    def heads(t, n):
        return t.view(1, -1, n, d).transpose(1, 2)
    h = norm.forward(x, mod[0], mod[1], torch.empty_like(x))
    close(h, norm64(x.double(), mod[0].double(), mod[1].double(), 1e-6, 1.0), 1, "norm")
    att = torch.empty_like(x)
    alloc = torch.tensor([1, 2, 4, 7], dtype=torch.uint8, device="cuda")
    plan.forward_projected(h, Wqkv, Wo, att, alloc=alloc, timesteps=[500.0], rotary=rotary, eps=1e-6)
    assert att.isfinite().all() and plan.device_status() == 0
    # (what the projected layer computes has tests of its own; here its output goes on)
    x1 = x + att
    h1 = norm.forward(x1, mod[2], mod[3], torch.empty_like(x1))
    q, k, v = heads(h1 @ Wq, H), heads(states[..., :G * d], G), heads(states[..., G * d:], G)      # (views of wider rows)
    out, lse = torch.empty_like(q), torch.empty(1, H, N, device="cuda")
    cross.forward(q, k, v, out, lse, lengths=lengths)
    x2 = x1 + out.transpose(1, 2).reshape(1, N, D)
    gate, up, y = (torch.empty(1, N, n, dtype=torch.bfloat16, device="cuda") for n in (2 * D, 2 * D, D))
    ffn.forward(x2, Wg, Wu, Wd, y, gate, up)

    # the second half backwards: block, cross attention, projection, norm
    dy = normal(1, N, D)
    dx2, dWg, dWu, dWd = torch.empty_like(x2), torch.empty_like(Wg), torch.empty_like(Wu), torch.empty_like(Wd)
    ffn.backward(x2, Wg, Wu, Wd, gate, up, dy, dx2, dWg, dWu, dWd)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    cross.backward(q, k, v, out, lse, heads(dx2, H), dq, dk, dv, lengths=lengths)
    dh1 = dq.transpose(1, 2).reshape(1, N, D) @ Wq.t()
    dx1, dscale, dshift = torch.empty_like(x1), torch.empty_like(mod[2]), torch.empty_like(mod[3])
    norm.backward(x1, mod[2], dh1, dx1, dscale, dshift)

    # the same in 64 bits from x1 on
    X, S, scale, shift, Q = (t.double().requires_grad_() for t in (x1, states, mod[2], mod[3], Wq))
    hr = norm64(X, scale, shift, 1e-6, 1.0)
    counts = torch.arange(K, device="cuda")[None] < lengths[:, None]
    o = cross64(heads(hr @ Q, H), *(heads(t, G).repeat_interleave(H // G, 1) for t in (S[..., :G * d], S[..., G * d:])), counts)
    X2 = X.detach() + o.transpose(1, 2).reshape(1, N, D)
    G_, U = X2 @ Wg.double(), X2 @ Wu.double()
    Y = (G_ * torch.sigmoid(G_) * U) @ Wd.double()
    close(h1, hr.detach(), 1, "second norm")
    close(heads(out.transpose(1, 2).reshape(1, N, D), H), o.detach(), 2, "cross attention")
    close(y, Y.detach(), 3, "block")
    gx, gs, gscale, gshift = torch.autograd.grad(Y, (X, S, scale, shift), dy.double())
    close(dx1, gx, 4, "dx")
    close(dk, heads(gs[..., :G * d], G), 4, "dk")
    close(dv, heads(gs[..., G * d:], G), 4, "dv")
    close(dscale, gscale, 4, "dscale")
    close(dshift, gshift, 4, "dshift")
    assert (dk[:, :, 61:] == 0).all() and cross.device_status() == 0 and ffn.device_status() == 0
