"""Rotary positions and the norm of queries and keys against their formulas in 64 bits.

Tolerances.  A result is rounded once: half a step, eps / 2 of its type relative to it.  Before that, in fp32:
  an angle is off by at most 2^-25 half turns (its conversion to a float) = 9.4e-8, sine and cosine by 2 units of 2^-24, each
  of the two products and their sum by 2^-24: below 5e-7 (|a| + |b|) m for either channel of a pair;
  r = 1 / sqrt(mean + eps): the sum of at most 256 squares in at most 32 + 5 additions one after the other, half of whose
  relative error (38 x 2^-24 = 2.3e-6) reaches r, and 2 units of the reciprocal root: below 1.4e-6; z = x r w adds 2 x 2^-24.
So a normed row is below 3e-6 (|z_a| + |z_b|) m off, a turned one below 5e-7 (|x_a| + |x_b|) m.  Backward: dz as a turned row;
n, g and the mean of g n (errors relative to the mean of |g n|, summed as above) give dx below 1e-5 r (|g| + |n| mean |g n|)
with |g| standing for both channels of the pair; dw below 1e-5 sum |dz n|, as up to 64 terms a thread, 6 in shuffles and
warps and 40 partial rows add 110 x 2^-24 = 6.6e-6 to the terms' own 3e-6."""
import math

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import RotaryConfig

pytestmark = pytest.mark.gpu
EPS = 1e-6


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rotate(cfg, handle, x, positions, inverse=False, absolute=False):
    """In 64 bits, pair by pair; positions [B or 1][N][axes].  absolute: |a| + |b| of each channel's pair instead."""
    theta, m = handle.frequencies()
    half = cfg.rot_dim // 2
    pairs = cfg.axis_pairs if any(cfg.axis_pairs) else (half, 0, 0)
    axis = torch.tensor([a for a, p in enumerate(pairs) for _ in range(p)], device=x.device)
    t = positions.double()[..., axis] * torch.tensor(theta, dtype=torch.float64, device=x.device)     # [B][N][half]
    t = t[:, None] * (-1 if inverse else 1)
    y = x.double().clone()
    i = torch.arange(half, device=x.device)
    ia, ib = (i, i + half) if cfg.layout == "half" else (2 * i, 2 * i + 1)
    a, b = y[..., ia].clone(), y[..., ib].clone()
    if absolute:
        y = y.abs()
        y[..., ia] = y[..., ib] = m * (a.abs() + b.abs())
    else:
        y[..., ia] = m * (a * t.cos() - b * t.sin())
        y[..., ib] = m * (a * t.sin() + b * t.cos())
    return y


def normed(x, w):
    x = x.double()
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS), None if w is None else w.double()


def given(cfg, positions, batch, tokens):
    if positions is not None:
        p = positions.reshape(-1, tokens, 3 if any(cfg.axis_pairs) else 1)
        return p.expand(batch, -1, -1)
    n = torch.arange(tokens, device="cuda")
    if any(cfg.axis_pairs):
        _, H, W = cfg.grid
        return torch.stack([n // (H * W), n // W % H, n % W], -1)[None]
    return n[None, :, None]


def within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert not torch.isnan(over).any(), what
    assert over.max().item() <= 0, f"{what}: {over.max().item():.3g} beyond the bound at {int(over.argmax())}"


def make(cfg, batch, heads, tokens, order, gen, offset=0, scale=1.0):
    """A tensor of head rows in one of several memory orders; `offset` elements into its storage."""
    d, dt = cfg.head_dim, torch.float32 if cfg.dtype == "fp32" else torch.bfloat16
    shape = {"heads_first": (batch, heads, tokens, d), "tokens_first": (batch, tokens, heads, d), "fused": (tokens, batch, heads, 3 * d),
             "padded": (batch, heads, tokens, d + 3)}[order]
    x = torch.randn(math.prod(shape) + offset, generator=gen, device="cuda")[offset:].view(shape).mul_(scale).to(dt)
    if offset:
        x = torch.cat([x.new_zeros(offset), x.flatten()])[offset:].view(shape)
    return {"heads_first": lambda: x, "tokens_first": lambda: x.transpose(1, 2), "fused": lambda: x[..., d:2 * d].permute(1, 2, 0, 3),
            "padded": lambda: x[..., :d]}[order]()


def check_forward(cfg, batch, heads, kv_heads, tokens, order="heads_first", positions=None, offset=0, weights=True, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    h = B.Rotary(cfg)
    q, k = (make(cfg, batch, n, tokens, order, gen, offset) for n in (heads, kv_heads))
    wq, wk = ((1 + 0.3 * torch.randn(cfg.head_dim, generator=gen, device="cuda")) if weights else None for _ in range(2))
    at = given(cfg, positions, batch, tokens)
    step = half_step(q.dtype)
    for inverse in (False, True):
        q2, k2 = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        h.apply(q, q2, k, k2, positions=positions, inverse=inverse)
        for x, y in ((q, q2), (k, k2)):
            want = rotate(cfg, h, x, at, inverse)
            within(y, want, step * want.abs() + 5e-7 * rotate(cfg, h, x, at, absolute=True), f"rotation, inverse {inverse}")
    q2, k2 = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    h.qk_norm(q, k, wq, wk, q2, k2, eps=EPS, positions=positions)
    for x, w, y in ((q, wq, q2), (k, wk, k2)):
        n, w = normed(x, w)
        z = n if w is None else n * w
        want = rotate(cfg, h, z, at)
        within(y, want, step * want.abs() + 3e-6 * rotate(cfg, h, z, at, absolute=True), "norm")


def check_backward(cfg, batch, heads, kv_heads, tokens, order="heads_first", positions=None, offset=0, weights=True, seed=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    h = B.Rotary(cfg)
    q, k, gq, gk = (make(cfg, batch, n, tokens, order, gen, offset) for n in (heads, kv_heads) * 2)
    wq, wk = ((1 + 0.3 * torch.randn(cfg.head_dim, generator=gen, device="cuda")) if weights else None for _ in range(2))
    at = given(cfg, positions, batch, tokens)
    dq, dk = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    dwq, dwk = (torch.full((cfg.head_dim,), float("nan"), device="cuda") for _ in range(2))
    h.qk_norm_backward(q, k, wq, wk, gq, gk, dq, dk, dwq, dwk, eps=EPS, positions=positions)
    for x, w, g, dx, dw in ((q, wq, gq, dq, dwq), (k, wk, gk, dk, dwk)):
        n, wd = normed(x, w)
        r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)
        dz, big = rotate(cfg, h, g, at, inverse=True), rotate(cfg, h, g, at, absolute=True)
        gz, gbig = (dz, big) if w is None else (dz * wd, big * wd.abs())
        want = r * (gz - n * (gz * n).mean(-1, keepdim=True))
        within(dx, want, half_step(x.dtype) * want.abs() + 1e-5 * r * (gbig + n.abs() * (gbig * n.abs()).mean(-1, keepdim=True)), "dx")
        within(dw, (dz * n).sum((0, 1, 2)), 1e-5 * (big * n.abs()).sum((0, 1, 2)), "dw")
    return h, (q, k, wq, wk, gq, gk, at)


CASES = [
    # every width of a row's pieces: 16, 8, 4 and 2 bytes (rot_dim / 2 = 64, 12, 10, 3), fp32: 16, 8, 4
    (RotaryConfig(128, 128), 2, 5, 2, 7, "heads_first"),
    (RotaryConfig(96, 24), 1, 3, 1, 33, "tokens_first"),
    (RotaryConfig(80, 20), 2, 2, 2, 5, "heads_first"),
    (RotaryConfig(64, 6), 1, 4, 1, 9, "tokens_first"),
    (RotaryConfig(256, 256, "fp32"), 1, 2, 1, 17, "tokens_first"),
    (RotaryConfig(80, 20, "fp32"), 1, 3, 3, 11, "heads_first"),
    (RotaryConfig(8, 2, "fp32"), 3, 1, 1, 1, "heads_first"),
    (RotaryConfig(256, 2), 1, 1, 1, 3, "heads_first"),
    (RotaryConfig(256, 254, "fp32"), 1, 2, 1, 3, "heads_first"),
    (RotaryConfig(128, 128, layout="interleaved"), 1, 9, 3, 40, "tokens_first"),
    (RotaryConfig(128, 72, layout="interleaved"), 1, 2, 1, 6, "heads_first"),
    (RotaryConfig(72, 18, layout="interleaved"), 2, 3, 1, 6, "heads_first"),
    (RotaryConfig(256, 250, "fp32", layout="interleaved"), 1, 2, 2, 5, "tokens_first"),
    (RotaryConfig(64, 64, axis_pairs=(8, 12, 12), grid=(3, 5, 7)), 2, 2, 1, 105, "heads_first"),
    (RotaryConfig(128, 96, "fp32", "interleaved", axis_pairs=(0, 40, 8), grid=(2, 4, 3)), 1, 2, 1, 24, "tokens_first"),
    (RotaryConfig(128, 128, scaling="by_parts", factor=16.0, original_length=4096), 1, 17, 4, 65, "fused"),
    # rows 2 x head_dim + 6 bytes apart: only single elements are aligned
    (RotaryConfig(32, 32), 2, 3, 1, 5, "padded"),
    (RotaryConfig(32, 32, "fp32", "interleaved"), 2, 3, 1, 4, "tokens_first"),
]


@pytest.mark.parametrize("cfg,batch,heads,kv,tokens,order", CASES)
def test_forward(cfg, batch, heads, kv, tokens, order):
    check_forward(cfg, batch, heads, kv, tokens, order)


@pytest.mark.parametrize("cfg,batch,heads,kv,tokens,order", CASES)
def test_backward(cfg, batch, heads, kv, tokens, order):
    check_backward(cfg, batch, heads, kv, tokens, order, weights=tokens != 6)


@pytest.mark.parametrize("offset", (1, 2, 4, 8))
def test_any_address(offset):
    """Tensors that start 2, 4, 8 or 16 bytes behind an aligned address."""
    check_forward(RotaryConfig(64, 32), 1, 3, 2, 6, offset=offset)
    check_backward(RotaryConfig(64, 32), 1, 3, 2, 6, offset=offset)


@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
def test_positions(dtype):
    """Given positions, per sample and shared, far ones, negative ones; single tokens and a batch of them."""
    cfg = RotaryConfig(128, 64, dtype, base=500000.0)
    p = torch.tensor([[0, 1, 2 ** 20 + 1, -7], [2 ** 31 - 1, -2 ** 31, 2 ** 24 + 1, 99999]], dtype=torch.int32, device="cuda")
    check_forward(cfg, 2, 2, 1, 4, positions=p)
    check_backward(cfg, 2, 2, 1, 4, positions=p)
    check_forward(cfg, 3, 2, 1, 4, positions=p[0].contiguous())
    check_forward(cfg, 100, 8, 2, 1, "tokens_first", positions=torch.randint(0, 10 ** 6, (100, 1), device="cuda").int())
    cfg = RotaryConfig(64, 64, dtype, axis_pairs=(8, 12, 12))
    check_forward(cfg, 2, 2, 2, 9, positions=torch.randint(-50, 200, (2, 9, 3), device="cuda").int())


def test_many_rows_and_heads():
    """More rows than a wave of blocks (the backward pass's blocks then walk on) and more heads than a block's 8; the same
    call twice gives the same bits."""
    cfg = RotaryConfig(64, 64)
    check_forward(cfg, 1, 21, 11, 3001)
    h, (q, k, wq, wk, gq, gk, _) = check_backward(cfg, 1, 21, 11, 3001)
    got = []
    for _ in range(2):
        d = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(wq), torch.empty_like(wk)]
        h.qk_norm_backward(q, k, wq, wk, gq, gk, *d, eps=EPS)
        got.append(d)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    check_backward(RotaryConfig(8, 8, "fp32"), 1, 700, 1, 2)        # more than 64 blocks of heads


def test_in_place_and_outside_rows():
    """Outputs that are their inputs give the same bits; what lies between the rows of a view stays."""
    cfg = RotaryConfig(64, 48)
    gen = torch.Generator("cuda").manual_seed(3)
    h = B.Rotary(cfg)
    store = torch.randn(2, 9, 5 * 64, generator=gen, device="cuda").to(torch.bfloat16)      # [batch][tokens][3 q | 1 k | 1 v heads]
    before = store.clone()
    q, k = store[:, :7, :192].unflatten(2, (3, 64)).transpose(1, 2), store[:, :7, 192:256].unflatten(2, (1, 64)).transpose(1, 2)
    w = torch.rand(64, generator=gen, device="cuda") + 0.5
    want = torch.empty_like(q), torch.empty_like(k)
    h.qk_norm(q, k, w, w, *want)
    h.qk_norm(q, k, w, w, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(store[..., 256:], before[..., 256:]) and torch.equal(store[:, 7:], before[:, 7:])
    # the gradient written over the gradient that came in
    g = torch.randn(2, 3, 7, 64, generator=gen, device="cuda").to(torch.bfloat16)
    d = torch.empty_like(g)
    h.qk_norm_backward(q, None, w, None, g, None, d, None)
    h.qk_norm_backward(q, None, w, None, g, None, g, None)
    assert torch.equal(d, g)


def test_without_keys_and_empty():
    cfg = RotaryConfig(64, 64)
    h = B.Rotary(cfg)
    x = torch.randn(1, 2, 5, 64, device="cuda").to(torch.bfloat16)
    y, z = torch.empty_like(x), torch.empty_like(x)
    h.apply(x, y)
    h.apply(x, z, x, torch.empty_like(x))
    assert torch.equal(y, z)
    e = x[:, :, :0]
    dw = torch.full((64,), 7.0, device="cuda")
    h.apply(e, e)
    h.qk_norm(e, None, None, None, e, None)
    h.qk_norm_backward(e, None, None, None, e, None, e, None, dw)
    assert not dw.any()
    one = torch.zeros_like(x)                                # rows of zeros: eps keeps them zeros
    h.qk_norm(one, None, None, None, y, None)
    assert not y.any()


def test_special_values():
    """Infinities and NaN stay in their row, and channels that are not turned are copied whatever stands beside them; rows whose squares
    leave fp32 are normed all the same; a broadcast input is read, a broadcast output refused."""
    cfg = RotaryConfig(64, 32, "fp32")
    h = B.Rotary(cfg)
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(1, 2, 6, 64, generator=gen, device="cuda")
    plain = torch.empty_like(x)
    h.apply(x, plain)
    bad = x.clone()
    bad[0, 0, 1, 40], bad[0, 0, 1, 3], bad[0, 1, 4, 50] = math.inf, math.nan, math.nan
    y = torch.empty_like(x)
    h.apply(bad, y)
    touched = torch.zeros_like(x, dtype=torch.bool)
    touched[0, 0, 1, 40] = touched[0, 0, 1, 3] = touched[0, 0, 1, 19] = touched[0, 1, 4, 50] = True
    assert torch.equal(y[~touched], plain[~touched])
    assert y[0, 0, 1, 40] == math.inf and y[0, 0, 1, 3].isnan() and y[0, 0, 1, 19].isnan() and y[0, 1, 4, 50].isnan()
    n = torch.empty_like(x)
    h.qk_norm(x, None, None, None, plain, None)
    h.qk_norm(bad, None, None, None, n, None)
    rows = [(0, 0, 1), (0, 1, 4)]
    for b, hd, t in ((b, hd, t) for b in range(1) for hd in range(2) for t in range(6)):
        assert torch.equal(n[b, hd, t], plain[b, hd, t]) == ((b, hd, t) not in rows)
    big = x * 2.0 ** 100                                     # a power of two: the same normed row, but for eps
    h.qk_norm(big, None, None, None, n, None, eps=1e-30)
    h.qk_norm(x, None, None, None, plain, None, eps=1e-30)
    within(n, plain.double(), 3e-6 * rotate(cfg, h, plain, given(cfg, None, 1, 6), absolute=True), "large rows")
    wide = x[:, :1].expand(1, 2, 6, 64)
    h.apply(wide, y)
    assert torch.equal(y[:, 0], y[:, 1])
    with pytest.raises(B.FFError):
        h.apply(x, wide)


def test_far_rows():
    """Rows that lie beyond 2^31 elements."""
    cfg = RotaryConfig(64, 64)
    h = B.Rotary(cfg)
    store = torch.zeros(2 ** 31 + 4096, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((2, 1, 2, 64), (2 ** 31 + 64, 64, 1024, 1))
    x.copy_(torch.randn(2, 1, 2, 64, device="cuda"))
    near, y = x.contiguous(), torch.empty(2, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    h.apply(near, y)
    h.apply(x, x)
    assert torch.equal(x, y) and int(store.count_nonzero()) <= 256


def test_gradient_against_differences():
    """dx and dw against central differences of the forward pass in fp32: the step 2^-6 leaves a third-order term below
    h^2 |f'''| / 6, and the outputs' rounding 2^-23 / 2^-6; together below 2e-3 of a gradient of size 1 .. 10."""
    cfg = RotaryConfig(32, 16, "fp32", axis_pairs=(2, 3, 3), grid=(1, 2, 2))
    h = B.Rotary(cfg)
    gen = torch.Generator("cuda").manual_seed(9)
    x, g = (torch.randn(1, 2, 4, 32, generator=gen, device="cuda") for _ in range(2))
    w = 1 + 0.3 * torch.randn(32, generator=gen, device="cuda")
    dx, dw, y = torch.empty_like(x), torch.empty_like(w), torch.empty_like(x)
    h.qk_norm_backward(x, None, w, None, g, None, dx, None, dw)

    def loss(x, w):
        h.qk_norm(x, None, w, None, y, None)
        return (y.double() * g.double()).sum().item()
    e = 2.0 ** -6
    for at in ((0, 0, 0, 0), (0, 1, 2, 9), (0, 0, 3, 15), (0, 1, 1, 20), (0, 1, 3, 31)):
        a, b = x.clone(), x.clone()
        a[at] += e
        b[at] -= e
        assert abs((loss(a, w) - loss(b, w)) / (2 * e) - dx[at].item()) < 2e-3
    for c in (0, 7, 8, 19, 31):
        a, b = w.clone(), w.clone()
        a[c] += e
        b[c] -= e
        assert abs((loss(x, a) - loss(x, b)) / (2 * e) - dw[c].item()) < 2e-3


def test_streams_and_graphs():
    """Calls on two streams at once and two captured graphs give what a call alone gives; a graph takes new inputs."""
    cfg = RotaryConfig(128, 128)
    h = B.Rotary(cfg)
    gen = torch.Generator("cuda").manual_seed(7)
    sets = []
    for _ in range(2):
        x, g = (torch.randn(1, 4, 2000, 128, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
        w = torch.rand(128, generator=gen, device="cuda") + 0.5
        sets.append((x, g, w, torch.empty_like(x), torch.empty_like(w)))

    def call(s):
        h.qk_norm_backward(s[0], None, s[2], None, s[1], None, s[3], None, s[4])
    want = []
    for s in sets:
        call(s)
        want.append((s[3].clone(), s[4].clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                call(s)
    torch.cuda.synchronize()
    assert all(torch.equal(s[3], a) and torch.equal(s[4], b) for s, (a, b) in zip(sets, want))
    graphs = []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(s)
        graphs.append(graph)
    for s in sets:
        s[3].zero_(), s[4].zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s[3], a) and torch.equal(s[4], b) for s, (a, b) in zip(sets, want))
    sets[0][0].copy_(sets[1][0]), sets[0][1].copy_(sets[1][1]), sets[0][2].copy_(sets[1][2])
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(sets[0][3], want[1][0]) and torch.equal(sets[0][4], want[1][1])


def test_binding_refusals():
    h = B.Rotary(RotaryConfig(64, 64))
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16, device="cuda")
    p = torch.arange(4, dtype=torch.int32, device="cuda")
    for call in (lambda: h.apply(x.float(), x), lambda: h.apply(x, x[:, :, :3]), lambda: h.apply(x.cpu(), x), lambda: h.apply(x, x, x),
                 lambda: h.apply(x[0], x[0]), lambda: h.apply(x[..., :32], x[..., :32]), lambda: h.apply(x.transpose(2, 3), x),
                 lambda: h.apply(x, x, positions=p.long()), lambda: h.apply(x, x, positions=p[:3]), lambda: h.apply(x, x, positions=p.cpu()),
                 lambda: h.qk_norm(x, None, torch.ones(63, device="cuda"), None, x, None), lambda: h.qk_norm(x, None, None, None, x, None, eps=0.0),
                 lambda: h.qk_norm(x, None, torch.ones(64), None, x, None), lambda: h.qk_norm(x, x, None, None, x, None),
                 lambda: h.qk_norm_backward(x, x, None, None, x, None, x, x)):
        with pytest.raises(B.FFError):
            call()


@pytest.mark.parametrize("tokens", (0, 1, 700))
def test_weight_gradient_without_keys(tokens):
    """dwk of a call without keys is a sum over no rows: zeros, and dwq as without it."""
    h = B.Rotary(RotaryConfig(64, 64))
    gen = torch.Generator("cuda").manual_seed(11)
    x, g = (torch.randn(1, 2, tokens, 64, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.rand(64, generator=gen, device="cuda") + 0.5
    dq, dwq, alone, dwk = torch.empty_like(x), *(torch.full((64,), 7.0, device="cuda") for _ in range(3))
    h.qk_norm_backward(x, None, w, None, g, None, dq, None, alone)
    h.qk_norm_backward(x, None, w, w, g, None, dq, None, dwq, dwk)
    assert not dwk.any() and torch.equal(dwq, alone)
    dwk.fill_(7.0)
    h.qk_norm_backward(x, None, w, None, g, None, dq, None, None, dwk)
    assert not dwk.any()


@pytest.mark.parametrize("eps", (1e30, 1e38))
def test_large_eps_beside_large_rows(eps):
    """Rows whose squares leave fp32, with an eps of the size of their mean (1e38) or far below it; rows of ordinary size with the same
    eps.  The mean and eps are added in fp32 as in any other row: the bounds of normed rows and of their gradients."""
    cfg = RotaryConfig(64, 32, "fp32")
    h = B.Rotary(cfg)
    gen = torch.Generator("cuda").manual_seed(12)
    x, g = (torch.randn(1, 2, 6, 64, generator=gen, device="cuda") for _ in range(2))
    x[:, :, ::2] *= 1e19
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(64, device="cuda")
    h.qk_norm(x, None, None, None, y, None, eps=eps)
    h.qk_norm_backward(x, None, None, None, g, None, dx, None, dw, eps=eps)
    at = given(cfg, None, 1, 6)
    r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + eps)
    n = x.double() * r
    want = rotate(cfg, h, n, at)
    within(y, want, half_step(x.dtype) * want.abs() + 3e-6 * rotate(cfg, h, n, at, absolute=True), "norm")
    dz, big = rotate(cfg, h, g, at, inverse=True), rotate(cfg, h, g, at, absolute=True)
    want = r * (dz - n * (dz * n).mean(-1, keepdim=True))
    within(dx, want, half_step(x.dtype) * want.abs() + 1e-5 * r * (big + n.abs() * (big * n.abs()).mean(-1, keepdim=True)), "dx")
    within(dw, (dz * n).sum((0, 1, 2)), 1e-5 * (big * n.abs()).sum((0, 1, 2)), "dw")


def test_special_values_backward():
    """A row of x or of the gradient that holds an infinity or a NaN spoils its own dx and, in the channels that the formula says, dw;
    the other rows keep their bits.  Rows whose squares leave fp32 have the gradient of the same rows scaled, divided by the scale."""
    cfg = RotaryConfig(64, 32, "fp32")
    h = B.Rotary(cfg)
    gen = torch.Generator("cuda").manual_seed(13)
    x, g = (torch.randn(1, 2, 70, 64, generator=gen, device="cuda") for _ in range(2))
    w = torch.rand(64, generator=gen, device="cuda") + 0.5
    at = given(cfg, None, 1, 70)

    def call(x, g, eps=EPS):
        dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
        h.qk_norm_backward(x, None, w, None, g, None, dx, None, dw, eps=eps)
        return dx, dw
    clean, _ = call(x, g)
    for into_x, value, channel in ((True, math.nan, 3), (True, math.inf, 40), (False, math.nan, 5), (False, -math.inf, 50), (False, math.inf, 20)):
        bad = [x.clone(), g.clone()]
        bad[0 if into_x else 1][0, 1, 66, channel] = value
        dx, dw = call(*bad)
        n, wd = normed(bad[0], w)
        r = 1 / torch.sqrt(bad[0].double().square().mean(-1, keepdim=True) + EPS)
        dz, big = rotate(cfg, h, bad[1], at, inverse=True), rotate(cfg, h, bad[1], at, absolute=True)
        want = r * (dz * wd - n * (dz * wd * n).mean(-1, keepdim=True))
        others = torch.ones(1, 2, 70, dtype=torch.bool, device="cuda")
        others[0, 1, 66] = False
        assert torch.equal(dx[others], clean[others])
        assert torch.equal(dx[0, 1, 66].isfinite(), want[0, 1, 66].isfinite())
        want, bound = (dz * n).sum((0, 1, 2)), 1e-5 * (big * n.abs()).sum((0, 1, 2))
        fine = want.isfinite()
        assert torch.equal(dw.isfinite(), fine)
        if fine.any():
            within(dw[fine], want[fine], bound[fine], "dw")
    plain, scaled = call(x, g, 1e-30), call(x * 2.0 ** 100, g, 1e-30)
    n, wd = normed(x, w)
    r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True))
    big = rotate(cfg, h, g, at, absolute=True)
    within(scaled[0].double() * 2.0 ** 100, plain[0].double(), 2e-5 * r * (big * wd + n.abs() * (big * wd * n.abs()).mean(-1, keepdim=True)), "dx of large rows")
    within(scaled[1], plain[1].double(), 2e-5 * (big * n.abs()).sum((0, 1, 2)), "dw of large rows")
