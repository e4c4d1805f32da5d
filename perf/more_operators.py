"""The rest of a video transformer's layer, as it is measured: layer norm with weights of the model or of the sample (forward
and backward pass), and cross attention of the video's tokens to an encoder's states of another length (forward and backward
pass, one query token and many).

`own` chooses between the plain form, in elementary torch operations of 32 bits, and the package's kernels.  `exact` gives
the same outputs in 64 bits, from the definitions; gradients by differentiation of the forward formula."""
import math

import torch

own = False

NORM, CROSS = "layer_norm", "cross_attention"
EPS = 1e-6


def _norm_case(name, direction, dtype, batch, tokens, dim, weights):
    c = {} if name is None else {"name": name}
    c.update(op=NORM, direction=direction, dtype=dtype, batch=batch, tokens=tokens, dim=dim, weights=weights)
    return c


def _cross_case(name, direction, batch, queries, keys, heads, kv_heads, head_dim, order="tokens_first", keys_used="all"):
    c = {} if name is None else {"name": name}
    c.update(op=CROSS, direction=direction, dtype="bf16", batch=batch, queries=queries, keys=keys, heads=heads, kv_heads=kv_heads,
             head_dim=head_dim, order=order, keys_used=keys_used)
    return c


def listed():
    return [
        # the next token of eight running sequences, weights and bias of the model
        _norm_case("norm_next_token", "forward", "bf16", 8, 1, 2048, "model"),
        # 64K tokens of a video grid; scale and shift of the sample, made from the diffusion timestep
        _norm_case("norm_grid_64k", "forward", "bf16", 1, 65536, 2048, "sample"),
        # fp32 rows of odd length
        _norm_case("norm_fp32_odd", "forward", "fp32", 1, 11000, 1155, "model"),
        # training on two short clips, gradients of each sample's scale and shift
        _norm_case("norm_back_clips", "backward", "bf16", 2, 8192, 1024, "sample"),
        # training of the model's own weights on an odd number of tokens
        _norm_case("norm_back_9999", "backward", "bf16", 1, 9999, 2048, "model"),
        # the next token of eight sequences, each with its own number of encoder states; grouped key heads
        _cross_case("cross_next_token", "forward", 8, 1, 4096, 32, 8, 128, keys_used="lengths"),
        # the 64K layer's 24 heads of 128 channels against 512 states of a text
        _cross_case("cross_grid_64k", "forward", 1, 65536, 512, 24, 24, 128),
        # training forward (the rows' log sums are kept): two clips, short captions with padding in between and behind
        _cross_case("cross_train_caption", "forward_train", 2, 8192, 77, 16, 16, 64, keys_used="mask"),
        # few queries against many states (latents that read an image's or a sound's states), 80 channels a head
        _cross_case("cross_long_states", "forward", 1, 1000, 9001, 12, 4, 80, order="heads_first"),
        # backward pass of a short clip, six heads
        _cross_case("cross_back_16k", "backward", 1, 16384, 512, 6, 6, 128),
        # ... of three padded samples of odd length with grouped keys
        _cross_case("cross_back_grouped", "backward", 3, 4097, 300, 16, 4, 64, keys_used="lengths"),
        # ... of the 64K layer
        _cross_case("cross_back_64k", "backward", 1, 65536, 512, 24, 24, 128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_norm(rng):
    dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
    dim = rng.choice((8 * _log_int(rng, 16, 640), 8 * _log_int(rng, 16, 640), _log_int(rng, 100, 5120)))
    return _norm_case(None, rng.choice(("forward", "backward")), dtype, rng.choice((1, 1, 2, 3, 8)), _log_int(rng, 1, 65536), dim,
                      rng.choice(("model", "sample")))


def _draw_cross(rng):
    kv_heads = rng.choice((1, 2, 4, 6, 8, 12))
    direction = rng.choice(("forward", "forward", "forward_train", "backward", "backward"))
    queries = rng.choice((1, rng.randint(2, 64))) if direction == "forward" and rng.random() < 0.4 else _log_int(rng, 64, 65536)
    return _cross_case(None, direction, rng.choice((1, 1, 2, 3, 8)), queries, _log_int(rng, 1, 10000), kv_heads * rng.choice((1, 1, 2, 4)),
                       kv_heads, rng.choice((32, 64, 64, 80, 96, 128, 128, 128)), rng.choice(("heads_first", "tokens_first")),
                       rng.choice(("all", "lengths", "mask")))


def _cost(case):
    w = work(case)
    return w["bytes"] / 6.4e12 + w["flops"] / 1.4e15


def draw(rng):
    """A case of the same ranges, no dearer than the largest listed one of its operator and direction."""
    kind = _draw_norm if rng.random() < 0.4 else _draw_cross
    while True:
        c = kind(rng)
        if _cost(c) <= max(_cost(x) for x in listed() if x["op"] == c["op"] and (x["direction"] == "backward") == (c["direction"] == "backward")):
            return c


def _lengths(case):
    """States that each sample has: from all of them down to a quarter."""
    B, K = case["batch"], case["keys"]
    return [max(1, K - 3 * K * b // (4 * B)) for b in range(B)] if case["keys_used"] == "lengths" else [K] * B


def work(case):
    """Bytes: inputs read once, outputs written once (of keys and values those that count).  Operations: of the norm eight a value,
    backward sixteen; of the attention its matrix products."""
    back = case["direction"] == "backward"
    if case["op"] == NORM:
        e = 4 if case["dtype"] == "fp32" else 2
        values = float(case["batch"]) * case["tokens"] * case["dim"]
        weights = case["dim"] * (case["batch"] if case["weights"] == "sample" else 1) * 4.0
        return {"bytes": (3 if back else 2) * values * e + (3 if back else 2) * weights, "flops": values * (16 if back else 8)}
    row, rows = case["head_dim"] * 2.0, float(case["batch"]) * case["queries"] * case["heads"]
    kept = float(sum(_lengths(case))) * (0.8 if case["keys_used"] == "mask" else 1.0)
    pairs = kept * case["queries"] * case["heads"]
    every = float(case["batch"]) * case["keys"] * case["kv_heads"] * row     # (gradients of all states, zeros among them)
    small = 4.0 * case["batch"] if case["keys_used"] == "lengths" else 1.0 * case["batch"] * case["keys"] if case["keys_used"] == "mask" else 0.0
    small += 4.0 * rows if case["direction"] != "forward" else 0.0
    if back:
        return {"bytes": 4 * rows * row + 2 * kept * case["kv_heads"] * row + 2 * every + small, "flops": 10 * pairs * case["head_dim"]}
    return {"bytes": 2 * rows * row + 2 * kept * case["kv_heads"] * row + small, "flops": 4 * pairs * case["head_dim"]}


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _heads_tensor(case, heads, tokens, gen, scale=1.0):
    """[batch][heads][tokens][head_dim] in bf16, in memory either so or token-major (a view of what a projection writes)."""
    B, d = case["batch"], case["head_dim"]
    shape = (B, heads, tokens, d) if case["order"] == "heads_first" else (B, tokens, heads, d)
    x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    for b in range(B):
        x[b].copy_(torch.randn(shape[1:], generator=gen, device="cuda") * scale)
    return x if case["order"] == "heads_first" else x.transpose(1, 2)


def _handle(case):
    from paper_2604_22808_b200 import binding, configs
    if case["op"] == NORM:
        return binding.LayerNorm(configs.LayerNormConfig(dim=case["dim"], dtype=case["dtype"], eps=EPS, unit_offset=case["weights"] == "sample"))
    return binding.CrossAttention(configs.CrossAttentionConfig(head_dim=case["head_dim"], heads=case["heads"], kv_heads=case["kv_heads"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = {"case": case}

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * scale
    if case["op"] == NORM:
        dtype, D = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16, case["dim"]
        shape, wshape = (case["batch"], case["tokens"], D), (case["batch"], D) if case["weights"] == "sample" else (D,)
        # a residual stream: channels of different sizes and means
        size, mean = torch.exp(0.5 * normal(D)), 0.5 * normal(D)
        s["x"] = torch.empty(shape, dtype=dtype, device="cuda")
        for b in range(case["batch"]):
            s["x"][b] = (normal(*shape[1:]) * size + mean).to(dtype)
        s["weight"], s["bias"] = normal(*wshape, scale=0.2) + (0.0 if case["weights"] == "sample" else 1.0), normal(*wshape, scale=0.2)
        s["y"] = torch.empty_like(s["x"])
        if case["direction"] == "backward":
            s["dy"] = normal(*shape).to(dtype)
            s["dweight"], s["dbias"] = torch.empty_like(s["weight"]), torch.empty_like(s["bias"])
    else:
        B, N, K, H, G = (case[k] for k in ("batch", "queries", "keys", "heads", "kv_heads"))
        s["q"], s["k"], s["v"] = _heads_tensor(case, H, N, gen, 1.5), _heads_tensor(case, G, K, gen), _heads_tensor(case, G, K, gen)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["keys_used"] == "lengths" else None
        s["mask"] = None
        if case["keys_used"] == "mask":
            s["mask"] = torch.rand(B, K, generator=gen, device="cuda") < 0.8
            s["mask"][:, 0] = True
        s["out"] = torch.empty_like(s["q"])                     # (keeps the order in memory)
        s["lse"] = torch.empty(B, H, N, dtype=torch.float32, device="cuda") if case["direction"] != "forward" else None
        if case["direction"] == "backward":
            s["dout"] = _heads_tensor(case, H, N, gen)
            out, lse = _plain_attention(s)                       # kept by the forward pass
            s["out"].copy_(out), s["lse"].copy_(lse)
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[k]) for k in "qkv")
    if own:
        s["handle"] = _handle(case)
    return s


# ---- plain form -----------------------------------------------------------------------------------------------------------
def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    w, b = (s[k][:, None] if case["weights"] == "sample" else s[k] for k in ("weight", "bias"))
    w = 1 + w if case["weights"] == "sample" else w
    c = x - x.mean(-1, keepdim=True)
    r = 1 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    if case["direction"] == "forward":
        return {"y": (c * r * w + b).to(s["x"].dtype)}
    n, dy = c * r, s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    over = 1 if case["weights"] == "sample" else (0, 1)
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * n).sum(over, dtype=torch.float64).float(), "dbias": dy.sum(over, dtype=torch.float64).float()}


def _left_out(case, s):
    """[batch][1][1][keys]: keys that do not count."""
    if s["mask"] is not None:
        return ~s["mask"][:, None, None, :]
    if s["lengths"] is not None:
        return (torch.arange(case["keys"], device="cuda") >= s["lengths"][:, None])[:, None, None, :]
    return None


def _per_group(t, G):
    """[batch][heads][tokens][...] as [batch][key heads][heads a key head * tokens][...]."""
    return t.reshape(t.shape[0], G, -1, *t.shape[3:])


def _plain_scores(s):
    case = s["case"]
    q, k = _per_group(s["q"].float(), case["kv_heads"]), s["k"].float()
    scores = (q @ k.transpose(-1, -2)) * case["head_dim"] ** -0.5
    gone = _left_out(case, s)
    return scores if gone is None else scores.masked_fill_(gone, -math.inf)


def _plain_attention(s):
    case = s["case"]
    scores = _plain_scores(s)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ s["v"].float()) / total
    return out.reshape(s["q"].shape).to(torch.bfloat16), (top + total.log()).reshape(case["batch"], case["heads"], case["queries"])


def _plain_attention_back(s):
    case = s["case"]
    G = case["kv_heads"]
    p = _plain_scores(s).sub_(_per_group(s["lse"], G)[..., None]).exp_()
    q, dout = _per_group(s["q"].float(), G), _per_group(s["dout"].float(), G)
    dv = p.transpose(-1, -2) @ dout
    delta = (dout * _per_group(s["out"].float(), G)).sum(-1, keepdim=True)
    ds = (dout @ s["v"].float().transpose(-1, -2)).sub_(delta).mul_(p).mul_(case["head_dim"] ** -0.5)
    dq, dk = ds @ s["k"].float(), ds.transpose(-1, -2) @ q
    return {"dq": dq.reshape(s["q"].shape).to(torch.bfloat16), "dk": dk.to(torch.bfloat16), "dv": dv.to(torch.bfloat16)}


# ---- the package's kernels ------------------------------------------------------------------------------------------------
def _own(s):
    case, h = s["case"], s["handle"]
    if case["op"] == NORM:
        if case["direction"] == "forward":
            h.forward(s["x"], s["weight"], s["bias"], s["y"])
            return {"y": s["y"]}
        h.backward(s["x"], s["weight"], s["dy"], s["y"], s["dweight"], s["dbias"])
        return {"dx": s["y"], "dweight": s["dweight"], "dbias": s["dbias"]}
    keys = {"lengths": s["lengths"], "mask": s["mask"]}
    if case["direction"] == "backward":
        h.backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], **keys)
        return {k: s[k] for k in ("dq", "dk", "dv")}
    h.forward(s["q"], s["k"], s["v"], s["out"], lse=s["lse"], **keys)
    return {"out": s["out"], "lse": s["lse"]} if case["direction"] == "forward_train" else {"out": s["out"]}


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["op"] == NORM:
        return _plain_norm(state)
    if case["direction"] == "backward":
        return _plain_attention_back(state)
    out, lse = _plain_attention(state)
    return {"out": out, "lse": lse} if case["direction"] == "forward_train" else {"out": out}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------------
def _exact_norm(case, s):
    x, w, b = (s[k].double().requires_grad_() for k in ("x", "weight", "bias"))
    sample = case["weights"] == "sample"
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    n = (x - mean) * (var + EPS).rsqrt()
    y = n * (1 + w).unsqueeze(1) + b.unsqueeze(1) if sample else n * w + b
    if case["direction"] == "forward":
        return {"y": y.detach()}
    return dict(zip(("dx", "dweight", "dbias"), torch.autograd.grad(y, (x, w, b), s["dy"].double())))


def _exact_head(case, s, b, h):
    """Output and log sum of one head of one sample, and the leaves they are made from."""
    g = h // (case["heads"] // case["kv_heads"])
    q, k, v = s["q"][b, h].double(), s["k"][b, g].double(), s["v"][b, g].double()
    if case["direction"] == "backward":
        q, k, v = (t.requires_grad_() for t in (q, k, v))
    if s["mask"] is not None:
        used = s["mask"][b].nonzero()[:, 0]
    else:
        used = torch.arange(_lengths(case)[b], device="cuda")
    scores = torch.einsum("nd,kd->nk", q / math.sqrt(case["head_dim"]), k[used])
    return torch.softmax(scores, -1) @ v[used], torch.logsumexp(scores, -1), (q, k, v)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == NORM:
        return _exact_norm(case, s)
    back = case["direction"] == "backward"
    if back:
        res = {"d" + n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"}
    else:
        res = {"out": torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")}
        if case["direction"] == "forward_train":
            res["lse"] = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b in range(case["batch"]):
        for h in range(case["heads"]):
            out, lse, leaves = _exact_head(case, s, b, h)
            if back:
                g = h // (case["heads"] // case["kv_heads"])
                dq, dk, dv = torch.autograd.grad(out, leaves, s["dout"][b, h].double())
                res["dq"][b, h] = dq
                res["dk"][b, g] += dk
                res["dv"][b, g] += dv
            else:
                res["out"][b, h] = out
                if "lse" in res:
                    res["lse"][b, h] = lse
    return res
