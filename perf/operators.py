"""The operators of a transformer layer around the attention path, as they are measured: rotary positions of queries and
keys, the norm of queries and keys for each head with the rotation in the same pass (and its backward pass), and the gated
feed-forward block (inference, training forward, backward).

`own` chooses between the plain form, in elementary torch operations of 32 bits (angles in 64), and the package's
kernels.  `exact` gives the same outputs in 64 bits, from the definitions: the rotation as a product of complex numbers,
gradients by differentiation of the forward formula."""
import math

import torch

own = False

ROTARY, NORM, FFN = "rotary", "qk_norm_rotary", "gated_ffn"
EPS = 1e-6


def _heads_case(name, op, direction, dtype, batch, tokens, heads, kv_heads, head_dim, rot_dim, layout, positions,
                order="heads_first", grid=(0, 0, 0), axis_pairs=(0, 0, 0), base=10000.0, scaling="none", factor=1.0,
                original_length=0, first=0):
    c = {} if name is None else {"name": name}
    c.update(op=op, direction=direction, dtype=dtype, batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads,
             head_dim=head_dim, rot_dim=rot_dim, layout=layout, positions=positions, order=order, T=grid[0], H=grid[1],
             W=grid[2], pairs_t=axis_pairs[0], pairs_h=axis_pairs[1], pairs_w=axis_pairs[2], base=base, scaling=scaling,
             factor=factor, original_length=original_length, first=first)
    return c


def _ffn_case(name, direction, tokens, dim, hidden, activation):
    c = {} if name is None else {"name": name}
    c.update(op=FFN, direction=direction, dtype="bf16", tokens=tokens, dim=dim, hidden=hidden, activation=activation)
    return c


def listed():
    return [
        # the next token of eight running sequences, far into a context extended sixteenfold; grouped key heads
        _heads_case("rotary_next_token", ROTARY, "forward", "bf16", 8, 1, 32, 8, 128, 128, "half", "own", "tokens_first",
                    base=500000.0, scaling="by_parts", factor=16.0, original_length=8192, first=100000),
        # 64K tokens of a video grid, 16 heads of 64 channels, pairs of neighbouring channels turned by t, h and w
        _heads_case("rotary_grid_64k", ROTARY, "forward", "bf16", 1, 65536, 16, 16, 64, 64, "interleaved", "grid",
                    grid=(16, 64, 64), axis_pairs=(8, 12, 12)),
        # gradients of queries and keys turned back: packed fp32 sequences, half of each head of 80 channels turned
        _heads_case("rotary_back_packed", ROTARY, "inverse", "fp32", 1, 11000, 12, 4, 80, 40, "half", "packed",
                    "tokens_first", scaling="linear", factor=4.0),
        # the next token of two sequences
        _heads_case("norm_next_token", NORM, "forward", "bf16", 2, 1, 16, 4, 128, 128, "half", "own", "tokens_first",
                    first=4000),
        # what stands between the projections and the attention forward of the 64K layer: 24 heads of 128 channels
        _heads_case("norm_grid_64k", NORM, "forward", "bf16", 1, 65536, 24, 24, 128, 128, "half", "grid",
                    grid=(16, 64, 64), axis_pairs=(16, 24, 24)),
        # its backward pass on a short clip, six heads of 16K tokens
        _heads_case("norm_back_16k", NORM, "backward", "bf16", 1, 16384, 6, 6, 128, 128, "half", "grid",
                    grid=(16, 32, 32), axis_pairs=(16, 24, 24)),
        # ... and in token-major training batches of odd length with grouped keys and a larger base
        _heads_case("norm_back_grouped", NORM, "backward", "bf16", 2, 8191, 32, 8, 128, 64, "interleaved", "row",
                    "tokens_first", scaling="ntk", factor=8.0),
        # one token through the block: every weight is read for one row
        _ffn_case("ffn_next_token", "forward", 1, 2048, 5632, "silu"),
        # a step of a few dozen sequences together
        _ffn_case("ffn_37_tokens", "forward", 37, 2048, 5632, "silu"),
        # all tokens of the paper's own 64K layer (16 heads of 64 channels)
        _ffn_case("ffn_grid_64k", "forward", 65536, 1024, 2816, "silu"),
        # training forward of a short clip: both projections are kept for the backward pass
        _ffn_case("ffn_train_16k", "forward_train", 16384, 768, 2056, "gelu_tanh"),
        # backward pass of an odd number of tokens
        _ffn_case("ffn_back_9999", "backward", 9999, 2048, 5632, "silu"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_heads(rng):
    op = rng.choice((ROTARY, NORM))
    direction = rng.choice(("forward", "inverse") if op == ROTARY else ("forward", "backward"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    head_dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
    layout = rng.choice(("half", "half", "interleaved"))
    order = rng.choice(("heads_first", "tokens_first"))
    kv_heads = rng.choice((1, 2, 4, 6, 8, 16))
    heads = kv_heads * rng.choice((1, 1, 2, 4))
    if rng.random() < 0.4:                      # a video grid
        grid = (rng.randint(1, 32), _log_int(rng, 4, 64), _log_int(rng, 4, 64))
        pt = max(1, head_dim // 8)
        ph = (head_dim // 2 - pt) // 2
        return _heads_case(None, op, direction, dtype, rng.choice((1, 1, 2)), math.prod(grid), heads, heads, head_dim,
                           2 * (pt + 2 * ph), layout, "grid", order, grid, (pt, ph, ph), base=rng.choice((256.0, 10000.0)))
    rot_dim = rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4))
    scaling = rng.choice(("none", "linear", "ntk", "by_parts"))
    positions = rng.choice(("own", "row", "packed"))
    tokens = rng.choice((1, 1, rng.randint(2, 9))) if positions == "own" else _log_int(rng, 1, 65536)
    batch = _log_int(rng, 1, 256) if positions == "own" else rng.choice((1, 1, 2, 3))
    return _heads_case(None, op, direction, dtype, batch, tokens, heads, kv_heads, head_dim, rot_dim, layout, positions,
                       order, base=rng.choice((10000.0, 500000.0)), scaling=scaling,
                       factor=1.0 if scaling == "none" else rng.choice((2.0, 4.0, 8.0, 16.0)),
                       original_length=rng.choice((2048, 4096, 8192)) if scaling == "by_parts" else 0,
                       first=_log_int(rng, 1, 500000) if positions == "own" else 0)


def _draw_ffn(rng):
    dim = 8 * _log_int(rng, 32, 256)
    hidden = 8 * _log_int(rng, 64, 704)
    direction = rng.choice(("forward", "forward", "forward_train", "backward"))
    tokens = _log_int(rng, 1, 256) if direction == "forward" and rng.random() < 0.5 else _log_int(rng, 1, 65536)
    return _ffn_case(None, direction, tokens, dim, hidden, rng.choice(("silu", "silu", "gelu_tanh", "gelu")))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.5e12 + w["flops"] / 1.4e15


def draw(rng):
    """A case of the same ranges, no dearer than the largest listed one of its operator's kind."""
    heads_like = rng.random() < 0.55
    kind = (ROTARY, NORM) if heads_like else (FFN,)
    most = max(_cost(c) for c in listed() if c["op"] in kind)
    while True:
        c = _draw_heads(rng) if heads_like else _draw_ffn(rng)
        if _cost(c) <= most:
            return c


def work(case):
    """Bytes: inputs read once, outputs written once (positions and the norms' weights too; where a grid gives the
    positions, nothing is read for them).  Operations: six per turned pair, four more per channel for a norm, twelve for its
    backward pass; the matrix products of the block."""
    if case["op"] == FFN:
        M, D, F = float(case["tokens"]), case["dim"], case["hidden"]
        weights = 3.0 * D * F * 2
        if case["direction"] == "forward":
            return {"bytes": weights + 2 * M * D * 2, "flops": 6 * M * D * F}
        if case["direction"] == "forward_train":
            return {"bytes": weights + 2 * M * D * 2 + 2 * M * F * 2, "flops": 6 * M * D * F}
        return {"bytes": 2 * weights + 3 * M * D * 2 + 2 * M * F * 2, "flops": 12 * M * D * F}
    e = 4 if case["dtype"] == "fp32" else 2
    rows = float(case["batch"]) * case["tokens"] * (case["heads"] + case["kv_heads"])
    values = rows * case["head_dim"]
    axes = 3 if case["pairs_t"] else 1
    given = {"grid": 0, "row": case["tokens"], "packed": case["tokens"], "own": case["batch"] * case["tokens"]}[case["positions"]]
    small = 4.0 * axes * given
    back = case["direction"] == "backward"
    flops = rows * (case["rot_dim"] // 2) * 6
    if case["op"] == NORM:
        small += 4.0 * 2 * case["head_dim"] * (2 if back else 1)
        flops += values * (12 if back else 4)
    return {"bytes": (3 if back else 2) * values * e + small, "flops": flops}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _heads_tensor(case, heads, gen, scale=None):
    """[batch][heads][tokens][head_dim], in memory either so or token-major (a view of what a projection writes)."""
    B, N, d = case["batch"], case["tokens"], case["head_dim"]
    shape = (B, heads, N, d) if case["order"] == "heads_first" else (B, N, heads, d)
    x = torch.empty(shape, dtype=_dtype(case), device="cuda")
    for b in range(B):
        v = torch.randn(shape[1:], generator=gen, device="cuda")
        x[b].copy_(v if scale is None else v * scale)
    return x if case["order"] == "heads_first" else x.transpose(1, 2)


def _positions(case, gen):
    B, N = case["batch"], case["tokens"]
    if case["positions"] == "grid":
        return None                                    # the token's index in the grid
    if case["positions"] == "row":
        return torch.arange(case["first"], case["first"] + N, dtype=torch.int32, device="cuda")
    if case["positions"] == "own":                     # every sample is somewhere else in its sequence
        start = torch.randint(case["first"], 2 * case["first"] + 1, (B, 1), generator=gen, device="cuda")
        return (start + torch.arange(N, device="cuda")).to(torch.int32).contiguous()
    cuts = torch.randint(0, N, (7,), generator=gen, device="cuda").sort().values     # eight sequences in a row
    at = torch.arange(N, device="cuda")
    begin = torch.cat([torch.zeros(1, dtype=cuts.dtype, device="cuda"), cuts])[torch.searchsorted(cuts, at, right=True)]
    return (at - begin).to(torch.int32).contiguous()


def _rotary_handle(case):
    from paper_2604_22808_b200 import binding, configs
    return binding.Rotary(configs.RotaryConfig(
        head_dim=case["head_dim"], rot_dim=case["rot_dim"], dtype=case["dtype"], layout=case["layout"], base=case["base"],
        scaling=case["scaling"], factor=case["factor"], original_length=case["original_length"],
        axis_pairs=(case["pairs_t"], case["pairs_h"], case["pairs_w"]), grid=(case["T"], case["H"], case["W"])))


def _ffn_handle(case):
    from paper_2604_22808_b200 import binding, configs
    return binding.GatedFFN(configs.FFNConfig(dim=case["dim"], hidden=case["hidden"], activation=case["activation"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}
    if case["op"] == FFN:
        M, D, F = case["tokens"], case["dim"], case["hidden"]

        def normal(*shape, scale=1.0):
            return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(torch.bfloat16)
        s["X"] = normal(M, D)
        s["Wg"], s["Wu"] = normal(D, F, scale=D ** -0.5), normal(D, F, scale=D ** -0.5)
        s["Wd"] = normal(F, D, scale=F ** -0.5)
        if case["direction"] == "backward":
            s["gate"], s["up"] = s["X"] @ s["Wg"], s["X"] @ s["Wu"]     # kept by the forward pass
            s["dout"] = normal(M, D, scale=0.1)
            s["results"] = [torch.empty_like(s[k]) for k in ("X", "Wg", "Wu", "Wd")]
        else:
            s["results"] = [torch.empty_like(s["X"])]
            if case["direction"] == "forward_train":
                s["results"] += [torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        if own:
            s["handle"] = _ffn_handle(case)
        return s
    # activations with channels of different sizes, as projections give them
    scale = torch.exp(0.5 * torch.randn(case["head_dim"], generator=gen, device="cuda"))
    s["q"], s["k"] = (_heads_tensor(case, h, gen, scale) for h in (case["heads"], case["kv_heads"]))
    s["positions"] = _positions(case, gen)
    if case["op"] == NORM:
        s["wq"], s["wk"] = (1.0 + 0.2 * torch.randn(case["head_dim"], generator=gen, device="cuda") for _ in range(2))
        if case["direction"] == "backward":
            s["dq_out"], s["dk_out"] = (_heads_tensor(case, h, gen) for h in (case["heads"], case["kv_heads"]))
            s["dwq"], s["dwk"] = torch.empty_like(s["wq"]), torch.empty_like(s["wk"])
    s["q_new"], s["k_new"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])      # (keep the order in memory)
    if own:
        s["handle"] = _rotary_handle(case)
    return s


# ---- plain form -----------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians per position of every pair, the axis that each pair turns with, and the magnitude of the rotation."""
    pairs = [p for p in (case["pairs_t"], case["pairs_h"], case["pairs_w"]) if p] or [case["rot_dim"] // 2]
    theta, axis = [], []
    for a, P in enumerate(pairs):
        base, i = case["base"], torch.arange(P, dtype=torch.float64, device="cuda")
        if case["scaling"] == "ntk" and P > 1:
            base = base * case["factor"] ** (P / (P - 1))
        t = base ** (-i / P)
        if case["scaling"] == "linear":
            t = t / case["factor"]
        elif case["scaling"] == "by_parts":            # few turns within the original length: interpolated; many: kept
            turns = case["original_length"] * t / (2 * math.pi)
            keep = ((turns - 1.0) / 31.0).clamp(0, 1)
            t = t * (keep + (1 - keep) / case["factor"])
        theta.append(t)
        axis.append(torch.full((P,), a, device="cuda"))
    magnitude = 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "by_parts" else 1.0
    return torch.cat(theta), torch.cat(axis), magnitude


def _angles(case, positions):
    """[batch or 1][1][tokens][pairs], in 64 bits."""
    theta, axis, magnitude = _frequencies(case)
    if positions is None:
        n = torch.arange(case["tokens"], device="cuda")
        H, W = case["H"], case["W"]
        at = torch.stack([n // (H * W), n // W % H, n % W], 1).double()[None]
        angle = at[:, :, axis] * theta
    else:
        angle = positions.double().reshape(-1, case["tokens"])[:, :, None] * theta
    return angle[:, None], magnitude


def _plain_turn(case, x, cos, sin):
    """x in 32 bits: the first rot_dim channels turned, the others as they are."""
    r = case["rot_dim"]
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _plain_heads(s):
    case = s["case"]
    angle, magnitude = _angles(case, s["positions"])
    cos, sin = (torch.cos(angle) * magnitude).float(), (torch.sin(angle) * magnitude).float()
    if case["direction"] != "forward":
        sin = -sin
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        if case["op"] == ROTARY:
            y = _plain_turn(case, x, cos, sin)
        else:
            w = s["w" + name]
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            if case["direction"] == "forward":
                y = _plain_turn(case, x * r * w, cos, sin)
            else:
                dz = _plain_turn(case, s["d" + name + "_out"].float(), cos, sin)
                out["dw" + name] = (dz * x * r).sum((0, 2)).sum(0)
                g = dz * w
                y = r * (g - x * r * r * (g * x).mean(-1, keepdim=True))
        out[name] = y.to(s[name].dtype)
    return out


def _plain_activation(name, g):
    """The activation and its derivative."""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)
    phi = 0.5 * (1 + torch.erf(g / math.sqrt(2)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def _plain_ffn(s):
    case = s["case"]
    X, Wg, Wu, Wd = (s[k].float() for k in ("X", "Wg", "Wu", "Wd"))
    if case["direction"] != "backward":
        gate, up = X @ Wg, X @ Wu
        out = {"out": ((_plain_activation(case["activation"], gate)[0] * up) @ Wd).to(torch.bfloat16)}
        if case["direction"] == "forward_train":
            out.update(gate=gate.to(torch.bfloat16), up=up.to(torch.bfloat16))
        return out
    gate, up, dout = (s[k].float() for k in ("gate", "up", "dout"))
    act, slope = _plain_activation(case["activation"], gate)
    dh = dout @ Wd.T
    dg, du = dh * up * slope, dh * act
    grads = {"dX": dg @ Wg.T + du @ Wu.T, "dWg": X.T @ dg, "dWu": X.T @ du, "dWd": (act * up).T @ dout}
    return {k: v.to(torch.bfloat16) for k, v in grads.items()}


# ---- the package's kernels ------------------------------------------------------------------------------------------------
def _own_heads(s):
    case, h = s["case"], s["handle"]
    if case["op"] == ROTARY:
        h.apply(s["q"], s["q_new"], s["k"], s["k_new"], positions=s["positions"], inverse=case["direction"] == "inverse")
    elif case["direction"] == "forward":
        h.qk_norm(s["q"], s["k"], s["wq"], s["wk"], s["q_new"], s["k_new"], eps=EPS, positions=s["positions"])
    else:
        h.qk_norm_backward(s["q"], s["k"], s["wq"], s["wk"], s["dq_out"], s["dk_out"], s["q_new"], s["k_new"], s["dwq"],
                           s["dwk"], eps=EPS, positions=s["positions"])
        return {"q": s["q_new"], "k": s["k_new"], "dwq": s["dwq"], "dwk": s["dwk"]}
    return {"q": s["q_new"], "k": s["k_new"]}


def _own_ffn(s):
    case, h, r = s["case"], s["handle"], s["results"]
    weights = s["Wg"], s["Wu"], s["Wd"]
    if case["direction"] == "backward":
        h.backward(s["X"], *weights, s["gate"], s["up"], s["dout"], dX=r[0], dWg=r[1], dWu=r[2], dWd=r[3])
        return dict(zip(("dX", "dWg", "dWu", "dWd"), r))
    if case["direction"] == "forward_train":
        h.forward(s["X"], *weights, r[0], gate=r[1], up=r[2])
        return dict(zip(("out", "gate", "up"), r))
    h.forward(s["X"], *weights, r[0])
    return {"out": r[0]}


def run(state):
    if state["case"]["op"] == FFN:
        return _own_ffn(state) if own else _plain_ffn(state)
    return _own_heads(state) if own else _plain_heads(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _exact_rotation(case, positions):
    """e^(i angle), times the magnitude: [batch or 1][1][tokens][pairs] complex numbers, one axis after the other."""
    s, kind = case["factor"], case["scaling"]
    if positions is None:
        places = torch.meshgrid(*(torch.arange(n, dtype=torch.float64, device="cuda") for n in (case["T"], case["H"], case["W"])), indexing="ij")
        axes = [(p.reshape(1, -1), n) for p, n in zip(places, (case["pairs_t"], case["pairs_h"], case["pairs_w"]))]
    else:
        axes = [(positions.to(torch.float64).reshape(-1, case["tokens"]), case["rot_dim"] // 2)]
    parts = []
    for place, P in axes:
        theta = []
        for i in range(P):
            t = math.exp(-math.log(case["base"]) * i / P)
            if kind == "ntk" and P > 1:
                t *= s ** (-i / (P - 1))
            elif kind == "linear":
                t /= s
            elif kind == "by_parts":
                turns = case["original_length"] * t / math.tau
                t *= 1.0 if turns >= 32 else 1 / s if turns <= 1 else ((turns - 1) + (32 - turns) / s) / 31
            theta.append(t)
        angle = place[..., None] * torch.tensor(theta, dtype=torch.float64, device="cuda")
        parts.append(torch.complex(angle.cos(), angle.sin()))
    return torch.cat(parts, -1)[:, None] * (1 + 0.1 * math.log(s) if kind == "by_parts" else 1)


def _exact_turn(case, x, turn):
    """Pairs as complex numbers, times e^(i angle)."""
    r = case["rot_dim"]
    p = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
    z = torch.view_as_real(torch.view_as_complex(p.contiguous()) * turn)
    z = z.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else z.flatten(-2)
    return torch.cat([z, x[..., r:]], -1)


def _exact_activation(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu_tanh":
        return g * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3))
    return g * 0.5 * torch.erfc(-g / math.sqrt(2))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == FFN:
        X, Wg, Wu, Wd = (s[k].double() for k in ("X", "Wg", "Wu", "Wd"))
        if case["direction"] != "backward":
            gate, up = X.matmul(Wg), X.matmul(Wu)
            out = {"out": (_exact_activation(case["activation"], gate) * up).matmul(Wd)}
            return {**out, "gate": gate, "up": up} if case["direction"] == "forward_train" else out
        gate, up = s["gate"].double().requires_grad_(), s["up"].double().requires_grad_()
        Wd.requires_grad_()
        out = (_exact_activation(case["activation"], gate) * up).matmul(Wd)
        dg, du, dWd = torch.autograd.grad(out, (gate, up, Wd), s["dout"].double())
        return {"dX": dg.matmul(Wg.t()) + du.matmul(Wu.t()), "dWg": X.t().matmul(dg), "dWu": X.t().matmul(du), "dWd": dWd}
    turn = _exact_rotation(case, s["positions"])
    if case["direction"] == "inverse":
        turn = turn.conj()
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        if case["op"] == ROTARY:
            out[name] = _exact_turn(case, x, turn)
            continue
        w = s["w" + name].double()
        back = case["direction"] == "backward"
        if back:
            x.requires_grad_(), w.requires_grad_()
        y = _exact_turn(case, x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["head_dim"] + EPS) * w, turn)
        if back:
            out[name], out["dw" + name] = torch.autograd.grad(y, (x, w), s["d" + name + "_out"].double())
        else:
            out[name] = y
    return out
