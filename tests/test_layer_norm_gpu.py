"""Layer norm against its formulas in 64 bits.

Tolerances, element by element, relative to sizes that belong to the row.  The mean of d values is d 2^-24 of their mean size off at
most (one rounding an addition; the sums run over pairs and threads, far fewer in a chain) and a value minus the mean another 2^-24;
so a centred value is off by e0 = (d + 2) 2^-24 times the row's mean size plus 2^-24 of itself.  The variance of centred values is
(d + 4) 2^-24 off relatively, its root half of that, the reciprocal root 2^-22: n = c r is below
(d + 40) 2^-24 (|n| + size r) off.  The result is rounded once: half a step of its type, 2^-8 (bf16) or 2^-24 (fp32)."""
import math

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import LayerNormConfig

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert not torch.isnan(over).any(), what
    assert over.max().item() <= 0, f"{what}: {over.max().item():.3g} beyond the bound at {int(over.argmax())}"


def normal(*shape, seed=0, scale=1.0, mean=0.0):
    return scale * torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed + sum(shape)), device="cuda") + mean


def reference(x, w, b, dy, plus, per_sample):
    """y, gradients, and what their errors are measured by."""
    d = x.shape[-1]
    X, DY = x.double(), dy.double()
    W = torch.ones(d, dtype=torch.float64, device="cuda") if w is None else w.double() + plus
    W = W[:, None] if w is not None and per_sample else W
    Bi = torch.zeros(d, dtype=torch.float64, device="cuda") if b is None else b.double()
    Bi = Bi[:, None] if b is not None and per_sample else Bi
    c = X - X.mean(-1, keepdim=True)
    r = ((c * c).mean(-1, keepdim=True) + EPS).rsqrt()
    n, g = c * r, DY * W
    k = (g * n).mean(-1, keepdim=True)
    m = g.mean(-1, keepdim=True)
    over = 1 if per_sample else tuple(range(x.dim() - 1))
    rel = (d + 40) * 2.0 ** -24
    en = rel * (n.abs() + X.abs().mean(-1, keepdim=True) * r)
    y = n * W + Bi
    ey = en * W.abs() + 2.0 ** -22 * ((n * W).abs() + y.abs())
    size = g.abs().mean(-1, keepdim=True)
    # g - m - n k: m and k are sums of d values, k of products with n
    ek = rel * (g * n).abs().mean(-1, keepdim=True) + (g.abs() * en).mean(-1, keepdim=True)
    dx = r * (g - m - n * k)
    ed = r * (rel * (size + g.abs()) + en * k.abs() + (n.abs() + en) * ek + 2.0 ** -22 * (n * k).abs()) + rel * dx.abs()
    rows = X.numel() // d // (x.shape[0] if per_sample else 1)
    add = (rows + 8) * 2.0 ** -24
    return {"y": (y, ey), "dx": (dx, ed), "dw": ((DY * n).sum(over), add * (DY * n).abs().sum(over) + (DY.abs() * en).sum(over)),
            "db": (DY.sum(over), add * DY.abs().sum(over))}


def check(dtype, shape, weights="model", plus=False, strided=False, scale=1.0, mean=0.0):
    d, t, half = shape[-1], TYPE[dtype], HALF[dtype]
    x, dy = (normal(*shape, seed=s, scale=c, mean=m).to(t) for s, c, m in ((1, scale, mean), (2, 1.0, 0.0)))
    per_sample = weights == "sample"
    w = b = None
    if weights != "none":
        wshape = (shape[0], d) if per_sample else (d,)
        w, b = normal(*wshape, seed=3, scale=0.3, mean=0.0 if plus else 1.0), normal(*wshape, seed=4)
    if strided:                                              # columns of wider rows, samples apart, nothing around them touched
        wide = torch.full((shape[0], shape[1] + 2, d + 24), float("nan"), dtype=t, device="cuda")
        place = slice(None), slice(1, 1 + shape[1]), slice(8, 8 + d)

        def put(v=None):
            s = wide.clone()
            if v is not None:
                s[place] = v
            return s, s[place]
    else:
        def put(v=None):
            s = torch.full_like(x, float("nan")) if v is None else v.clone()
            return s, s
    (xs, xv), (gs, gv), (ys, yv), (ds, dv) = put(x), put(dy), put(), put()
    norm = B.LayerNorm(LayerNormConfig(d, dtype, EPS, plus))
    assert norm.forward(xv, w, b, yv) is yv
    dw, db = (torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))) if w is not None else (None, None)
    norm.backward(xv, w, gv, dv, dw, db)
    want = reference(x, w, b, dy, float(plus), per_sample)
    for got, name in ((yv, "y"), (dv, "dx")):
        value, e = want[name]
        within(got, value, half * value.abs() + (1 + half) * e, name)
    if w is not None:
        within(dw, *want["dw"], "dweight"), within(db, *want["db"], "dbias")
    # again, over its own inputs: the same bits
    (_, y2), (_, g2) = put(x), put(dy)
    norm.forward(y2, w, b, y2)
    norm.backward(xv, w, g2, g2, None, None)
    assert torch.equal(y2, yv) and torch.equal(g2, dv)
    if strided:
        for s in (ys, ds):
            s[place] = float("nan")
            assert s.isnan().all()


@pytest.mark.parametrize("dim", [1, 2, 3, 8, 31, 64, 250, 256, 264, 513, 1024, 1032, 1155, 2048, 2050, 2056, 4104, 5120, 8191, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_row_lengths(dtype, dim):
    check(dtype, (3, 7, dim))


@pytest.mark.parametrize("shape", [(1, 1, 768), (1, 4000, 96), (5, 131, 320), (700, 1, 128), (3, 300, 2048), (9, 512), (1, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows(dtype, shape):
    check(dtype, shape)


@pytest.mark.parametrize("weights,plus", [("none", False), ("none", True), ("model", True), ("sample", False), ("sample", True)])
@pytest.mark.parametrize("shape", [(1, 50, 200), (3, 41, 1096), (650, 2, 72), (2, 600, 33)])
def test_weights(weights, plus, shape):
    check("bf16", shape, weights, plus)
    check("fp32", shape, weights, plus)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("bf16", 130), ("bf16", 131), ("bf16", 4096), ("fp32", 128), ("fp32", 1155)])
def test_strides(dtype, dim):
    check(dtype, (2, 9, dim), "sample", True, strided=True)


def test_mean_far_from_zero():
    """The variance is of centred values: a mean of a thousand deviations costs what its own rounding costs."""
    check("fp32", (2, 30, 1000), mean=1000.0)
    check("fp32", (2, 30, 700), scale=1e-3, mean=3.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [96, 129, 1024, 3000])
def test_rows_whose_squares_leave_fp32(dtype, dim):
    x = normal(4, dim).to(TYPE[dtype])
    big = x.clone()
    big[1] = x[1] * 2.0 ** 100
    big[2] = (x[2] * 2.0 ** 125).clamp(-3e38, 3e38)
    norm, y = B.LayerNorm(LayerNormConfig(dim, dtype, EPS)), torch.empty_like(x)
    norm.forward(big, None, None, y)
    X = big.double()
    c = X - X.mean(-1, keepdim=True)
    n = c * ((c * c).mean(-1, keepdim=True) + EPS).rsqrt()
    size = X.abs().mean(-1, keepdim=True) / ((c * c).mean(-1, keepdim=True) + EPS).sqrt()
    within(y, n, HALF[dtype] * n.abs() + 2 * (dim + 40) * 2.0 ** -24 * (n.abs() + size), "y")
    dy, dx = normal(4, dim, seed=9).to(TYPE[dtype]), torch.empty_like(x)
    dw, db = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    norm.backward(big, None, dy, dx, dw, db)
    want = (dy.double() * n).sum(0)
    within(dw, want, 4 * (dim + 50) * 2.0 ** -24 * (dy.double().abs() * (n.abs() + size)).sum(0), "dweight")
    assert dx.isfinite().all() and (dx[1:3].abs() <= 1e-20).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dim", [64, 1023, 4096])
def test_a_row_that_is_not_finite_spoils_itself_alone(value, dim):
    x = normal(6, dim).to(torch.bfloat16)
    norm, y, clean = B.LayerNorm(LayerNormConfig(dim)), torch.empty_like(x), torch.empty_like(x)
    norm.forward(x, None, None, clean)
    x[3, dim // 2] = value
    norm.forward(x, None, None, y)
    assert y[3].isnan().all()
    keep = [0, 1, 2, 4, 5]
    assert torch.equal(y[keep], clean[keep])


def test_shared_rows_and_no_rows():
    """Inputs with strides of zero are read as often as they stand there; sums over no rows are zeros."""
    d = 192
    one, w = normal(1, 1, d).to(torch.bfloat16), normal(d, seed=5)
    norm = B.LayerNorm(LayerNormConfig(d, eps=EPS))
    x, dy = one.expand(3, 5, d), normal(3, 5, d, seed=6).to(torch.bfloat16)
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(w), torch.empty_like(w)
    norm.forward(x, w, None, y)
    norm.backward(x, w, dy, dx, dw, db)
    y2, dx2, dw2, db2 = torch.empty_like(dy), torch.empty_like(dy), torch.empty_like(w), torch.empty_like(w)
    norm.forward(x.contiguous(), w, None, y2)
    norm.backward(x.contiguous(), w, dy, dx2, dw2, db2)
    assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2) and torch.equal(db, db2)
    for shape, wshape in (((0, d), (d,)), ((2, 0, d), (2, d)), ((0, 4, d), (d,))):
        x = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        w, dw, db = (torch.full(wshape, float("nan"), device="cuda") for _ in range(3))
        norm.forward(x, w, w, x)
        norm.backward(x, w, x, x, dw, db)
        assert (dw == 0).all() and (db == 0).all()


def test_some_of_the_gradients():
    d = 520
    x, dy, w = normal(3, 70, d).to(torch.bfloat16), normal(3, 70, d, seed=1).to(torch.bfloat16), normal(3, d, seed=2)
    norm = B.LayerNorm(LayerNormConfig(d))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    norm.backward(x, w, dy, dx, dw, db)
    for mask in range(8):
        got = [torch.full_like(t, float("nan")) if mask >> i & 1 else None for i, t in enumerate((dx, dw, db))]
        norm.backward(x, w, dy, *got)
        for g, t in zip(got, (dx, dw, db)):
            assert g is None or torch.equal(g, t)


def test_gradient_against_differences():
    d = 37
    x, w, b, dy = normal(2, 3, d), normal(2, d, seed=1), normal(2, d, seed=2), normal(2, 3, d, seed=3)
    norm = B.LayerNorm(LayerNormConfig(d, "fp32", 0.1, True))
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    norm.backward(x, w, dy, dx, dw, db)

    def loss(x, w, b):
        y = torch.empty_like(x)
        norm.forward(x, w, b, y)
        return (y.double() * dy.double()).sum().item()
    h = 2.0 ** -6          # (off by h^2 / 6 times a third derivative below 1e3, and 2^-22 of the loss's terms over 2 h)
    for i, (t, g) in enumerate(((x, dx), (w, dw), (b, db))):
        for at in (0, 17, t.numel() - 1):
            ends = []
            for s in (h, -h):
                args = [x, w, b]
                args[i] = t.clone()
                args[i].view(-1)[at] += s
                ends.append(loss(*args))
            assert abs((ends[0] - ends[1]) / (2 * h) - g.view(-1)[at].item()) < 2e-2 * (1 + g.abs().max().item())


def test_streams_and_graphs():
    """A call on a stream of its own, and captured calls that share a handle, each with its own workspace."""
    d = 1000
    norm = B.LayerNorm(LayerNormConfig(d))
    sets = []
    for s in range(2):
        x, dy = normal(2, 200, d, seed=s).to(torch.bfloat16), normal(2, 200, d, seed=10 + s).to(torch.bfloat16)
        sets.append((x, normal(d, seed=20 + s), dy, torch.empty_like(x), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")))
    for t in sets:
        norm.backward(*t)
    want = [[u.clone() for u in t[3:]] for t in sets]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for t in sets:
            norm.backward(*t)
            norm.forward(t[0], t[1], t[1], t[3])
            norm.backward(*t)
    for _ in range(2):
        for t in sets:
            for u in t[3:]:
                u.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for t, w in zip(sets, want) for u, v in zip(t[3:], w))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for u in sets[0][3:]:
            u.fill_(float("nan"))
        norm.backward(*sets[0])
    side.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(sets[0][3:], want[0]))


def test_many_rows_of_few_values():
    """Row offsets beyond 2^31 elements."""
    n, d = (1 << 31) // 4096 + 77, 4096
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    x[:] = normal(1, d).to(torch.bfloat16)
    x[-1] = normal(1, d, seed=1).to(torch.bfloat16)[0]
    y = torch.empty_like(x)
    norm = B.LayerNorm(LayerNormConfig(d))
    norm.forward(x, None, None, y)
    first, last = torch.empty(1, d, dtype=torch.bfloat16, device="cuda"), torch.empty(1, d, dtype=torch.bfloat16, device="cuda")
    norm.forward(x[:1], None, None, first)
    norm.forward(x[-1:], None, None, last)
    assert torch.equal(y[-1:], last) and bool((y[:-1] == first).all())
