"""A layer of all its parts: projections, norm and rotation of queries and keys, the attention forward, the output projection, the
gated feed-forward block."""
import numpy as np
import pytest
import torch

import harness as Hn
from oracle import freqformer_oracle as O
from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200 import configs as C
from paper_2604_22808_b200 import inputs as I
from paper_2604_22808_b200.configs import FFNConfig, RotaryConfig
from test_ffn_gpu import forward_bounds, within

pytestmark = pytest.mark.gpu
CFG = C.R_PAPER_REF.scaled("layer", T=16, H=16, W=16, low_cut=(8, 8, 8), mid_cut=(13, 13, 13), s=7)
EPS = 1e-6


def turned(x, cfg, rot, theta, w):
    """Oracle's [heads, T, H, W, d] rows: normed (w given), turned by the grid's positions, rounded to bf16; 64 bits."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + EPS) * w
    at = np.stack(np.meshgrid(*(np.arange(n) for n in cfg.grid), indexing="ij"), -1)
    axis = np.repeat(np.arange(3), rot.axis_pairs)
    t = at[..., axis] * theta
    half = rot.rot_dim // 2
    a, b = x[..., :half], x[..., half:rot.rot_dim]
    y = np.concatenate([a * np.cos(t) - b * np.sin(t), a * np.sin(t) + b * np.cos(t), x[..., rot.rot_dim:]], -1)
    return O.round_bf16(y)


@pytest.mark.parametrize("norm", (True, False))
def test_layer(norm):
    cfg, D = CFG, CFG.heads * CFG.head_dim
    rot = RotaryConfig(cfg.head_dim, 48, axis_pairs=(4, 10, 10), grid=cfg.grid, base=256.0)
    rotary = B.Rotary(rot)
    theta, _ = rotary.frequencies()
    X, (Wqkv, Wo) = I.layer_input(cfg), I.projection_weights(cfg)
    weights, U = I.router_weights(cfg), I.summary_projection(cfg)
    alloc = [1, 2, 4, 7]
    gen = np.random.default_rng(3)
    wq, wk = ((1 + 0.2 * gen.standard_normal(cfg.head_dim)).astype(np.float32) if norm else None for _ in range(2))
    q, k, v = O.project_qkv(X[0], Wqkv, cfg.heads, cfg.grid)
    ref = O.forward_sample(cfg, turned(q, cfg, rot, theta, wq), turned(k, cfg, rot, theta, wk), v, weights, U, cfg.timesteps[0], alloc=alloc)
    want = O.project_out(O.round_bf16(ref["out"]), Wo)

    def dev(a, dtype=torch.bfloat16):
        return None if a is None else torch.from_numpy(a).to("cuda", dtype)
    plan = B.Plan(cfg, weights, host_staging=True)
    x, wqkv, wo, masks = dev(X), dev(Wqkv), dev(Wo), torch.tensor(alloc, dtype=torch.uint8, device="cuda")
    kw = dict(rotary=rotary, wq=dev(wq, torch.float32), wk=dev(wk, torch.float32), eps=EPS if norm else 0.0)
    ffn = B.GatedFFN(FFNConfig(D, 696))
    g = torch.Generator("cuda").manual_seed(1)
    Wg, Wu, Wd = ((torch.randn(*s, generator=g, device="cuda") * s[0] ** -0.5).to(torch.bfloat16) for s in ((D, 696), (D, 696), (696, D)))
    out, y = torch.empty_like(x), torch.empty_like(x)

    def layer():
        plan.forward_projected(x, wqkv, wo, out, alloc=masks, **kw)
        h = x + out
        ffn.forward(h, Wg, Wu, Wd, y)
        return h + y
    got = layer()
    assert plan.device_status() == 0 and ffn.device_status() == 0
    assert plan.last_launches() == plain_launches(plan, x, wqkv, wo, masks) + 1
    # (the bounds of the projected layer without a rotation: what is turned is rounded to bf16 like the projections)
    plan.forward_projected(x, wqkv, wo, out, alloc=masks, **kw)
    Hn.assert_close(out[0].float().cpu().numpy(), want, "bf16", "turned layer", tol_scale=1.5)
    h = (x + out)[0]
    within(y[0], *forward_bounds("silu", h, Wg, Wu, Wd)[0], "feed-forward")
    # positions given instead of the grid's; a captured layer
    at = torch.from_numpy(np.stack(np.meshgrid(*(np.arange(n) for n in cfg.grid), indexing="ij"), -1).reshape(-1, 3)).to("cuda", torch.int32)
    again = torch.empty_like(out)
    plan.forward_projected(x, wqkv, wo, again, alloc=masks, positions=at.contiguous(), **kw)
    assert torch.equal(again, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer()
    out.zero_(), y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(captured, got)
    plan.destroy()


def plain_launches(plan, x, wqkv, wo, masks):
    plan.forward_projected(x, wqkv, wo, torch.empty_like(x), alloc=masks)
    return plan.last_launches()


def test_refusals():
    cfg = CFG
    plan = B.Plan(cfg, I.router_weights(cfg), host_staging=True)
    D = cfg.heads * cfg.head_dim
    x, w = torch.zeros(1, cfg.N, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, D, D, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(cfg.head_dim, device="cuda")
    good = RotaryConfig(64, 64)

    def call(rot, **kw):
        plan.forward_projected(x, w[:3], w[3], torch.empty_like(x), timesteps=[1.0], rotary=None if rot is None else B.Rotary(rot), **kw)
    call(good)
    for rot, kw in ((RotaryConfig(128, 64), {}), (RotaryConfig(64, 64, "fp32"), {}), (RotaryConfig(64, 64, axis_pairs=(8, 12, 12)), {}),
                    (RotaryConfig(64, 64, axis_pairs=(8, 12, 12), grid=(16, 16, 8)), {}), (good, dict(wq=one)), (good, dict(eps=-1.0)),
                    (good, dict(eps=float("nan"))), (good, dict(eps=1e-6, wk=one[:32])), (None, dict(wq=one)), (None, dict(eps=1e-6)),
                    (good, dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda")))):
        with pytest.raises(B.FFError):
            call(rot, **kw)
    lib = B.library()
    assert lib.ff_forward_projected_rotary(plan.handle, *[x.data_ptr()] * 3, None, None, 0, None, None, 0.0, None, None, x.data_ptr(), None) != 0
    assert lib.ff_forward_projected_rotary(None, *[None] * 5, 0, None, None, 0.0, None, None, None, None) == 1
    plan.destroy()


def test_positions_of_each_sample():
    # samples do not enter each other's sums: each must be what the same call gives it with its positions for both
    cfg = CFG.scaled("layer_pair", batch=2)
    rotary = B.Rotary(RotaryConfig(cfg.head_dim, 48))
    weights = I.router_weights(cfg)
    plan = B.Plan(cfg, weights, host_staging=True)
    X, (Wqkv, Wo) = I.layer_input(cfg), I.projection_weights(cfg)
    x, wqkv, wo = (torch.from_numpy(a).to("cuda", torch.bfloat16) for a in (X, Wqkv, Wo))
    masks = torch.tensor([1, 2, 4, 7] * 2, dtype=torch.uint8, device="cuda")
    one = torch.arange(cfg.N, dtype=torch.int32, device="cuda")
    two = one.flip(0).contiguous()

    def call(positions):
        return plan.forward_projected(x, wqkv, wo, torch.empty_like(x), alloc=masks, rotary=rotary, eps=EPS, positions=positions).clone()
    first, second, both = call(one), call(two), call(torch.stack((one, two)))
    assert plan.device_status() == 0
    assert not torch.equal(first[1], second[1])
    assert torch.equal(both[0], first[0]) and torch.equal(both[1], second[1])
    assert torch.equal(call(None), first)
    plan.destroy()
