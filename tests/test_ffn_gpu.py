"""The gated feed-forward block against its formulas in 64 bits.

Tolerances, element by element.  A result, and every operand kept between two products, is rounded to bf16 once: 2^-8 relative.
A sum of K products in fp32 is below K 2^-22 off, relative to the sum of the products' sizes (2^-23 for every addition, whichever way the
tensor core cuts).  The activation and its derivative are below 1e-5 (1 + |g|) off absolutely (exponential and reciprocal, 2^-21
relative, its argument's rounding |g| 2^-23 in front), and their slopes below 1.2 and 2.  What goes into a product reaches its result
through the other operand's sizes."""
import ctypes as C
import math

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import FFNConfig

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8


def summed(K):
    return K * 2.0 ** -22


def act(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    return 0.5 * g * (1 + torch.erf(g / math.sqrt(2)))


def act_and_slope(name, g):
    g = g.detach().clone().requires_grad_()
    a = act(name, g)
    return a.detach(), torch.autograd.grad(a.sum(), g)[0]


def within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert not torch.isnan(over).any(), what
    assert over.max().item() <= 0, f"{what}: {over.max().item():.3g} beyond the bound at {int(over.argmax())}"


def inputs(M, D, F, seed=0, scale=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)

    def normal(*shape, s=1.0):
        return (s * torch.randn(*shape, generator=gen, device="cuda")).to(torch.bfloat16)
    return normal(M, D, s=scale), normal(D, F, s=D ** -0.5), normal(D, F, s=D ** -0.5), normal(F, D, s=F ** -0.5), normal(M, D)


def nan_like(*shape):
    """A bf16 tensor of that shape, all NaN, in front of rows that must stay NaN (the second result says so)."""
    n = math.prod(shape)
    store = torch.full((n + 4096,), float("nan"), dtype=torch.bfloat16, device="cuda")
    return store[:n].view(shape), lambda: bool(store[n:].isnan().all())


def forward_bounds(activation, X, Wg, Wu, Wd):
    X, Wg, Wu, Wd = (t.double() for t in (X, Wg, Wu, Wd))
    D, F = Wg.shape
    g, u = X @ Wg, X @ Wu
    eg, eu = summed(D) * (X.abs() @ Wg.abs()), summed(D) * (X.abs() @ Wu.abs())
    a = act(activation, g)
    h = a * u
    ea = 1.2 * eg + 1e-5 * (1 + g.abs())
    eh = STEP * h.abs() + (1 + STEP) * (ea * u.abs() + a.abs() * eu + ea * eu)
    out = h @ Wd
    eo = eh @ Wd.abs() + summed(F) * ((h.abs() + eh) @ Wd.abs())
    return (out, STEP * out.abs() + (1 + STEP) * eo), (g, STEP * g.abs() + 2 * eg), (u, STEP * u.abs() + 2 * eu)


def check_forward(M, D, F, activation, keep, scale=1.0):
    X, Wg, Wu, Wd, _ = inputs(M, D, F, scale=scale)
    ffn = B.GatedFFN(FFNConfig(D, F, activation))
    out, clean = nan_like(M, D)
    gate, gate_clean = nan_like(M, F)
    up, up_clean = nan_like(M, F)
    ffn.forward(X, Wg, Wu, Wd, out, *((gate, up) if keep else ()))
    assert ffn.device_status() == 0
    want = forward_bounds(activation, X, Wg, Wu, Wd)
    within(out, *want[0], "out")
    if keep:
        within(gate, *want[1], "gate")
        within(up, *want[2], "up")
    assert clean() and gate_clean() and up_clean()


def check_backward(M, D, F, activation, seed=0):
    X, Wg, Wu, Wd, dout = inputs(M, D, F, seed)
    gate, up = X @ Wg, X @ Wu
    ffn = B.GatedFFN(FFNConfig(D, F, activation))
    (dX, c0), (dWg, c1), (dWu, c2), (dWd, c3) = nan_like(M, D), nan_like(D, F), nan_like(D, F), nan_like(F, D)
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX, dWg, dWu, dWd)
    assert ffn.device_status() == 0
    x, wg, wu, wd, g, u, do = (t.double() for t in (X, Wg, Wu, Wd, gate, up, dout))
    a, slope = act_and_slope(activation, g)
    ea = 1e-5 * (1 + g.abs())
    dh = do @ wd.T
    edh = summed(D) * (do.abs() @ wd.abs().T)
    dg, du, h = dh * u * slope, dh * a, a * u
    edg = STEP * dg.abs() + (1 + STEP) * u.abs() * (edh * (slope.abs() + ea) + dh.abs() * ea)
    edu = STEP * du.abs() + (1 + STEP) * (edh * (a.abs() + ea) + dh.abs() * ea)
    eh = STEP * h.abs() + (1 + STEP) * ea * u.abs()

    def product(pairs, K):
        """sum of A B over the pairs ((A, error of A), B), and its bound"""
        y = sum(A @ Bm for (A, _), Bm in pairs)
        e = sum(E @ Bm.abs() + summed(K) * ((A.abs() + E) @ Bm.abs()) for (A, E), Bm in pairs)
        return y, STEP * y.abs() + (1 + STEP) * e
    within(dX, *product([((dg, edg), wg.T), ((du, edu), wu.T)], 2 * F), "dX")
    for got, (v, e), name in ((dWg, (dg, edg), "dWg"), (dWu, (du, edu), "dWu")):
        y, e = product([((v.T, e.T), x)], M)
        within(got, y.T, e.T, name)
    within(dWd, *product([((h.T, eh.T), do)], M), "dWd")
    assert c0() and c1() and c2() and c3()


SIZES = [(1, 8, 8), (1, 256, 520), (2, 64, 64), (9, 72, 136), (16, 512, 128), (17, 1024, 264), (33, 200, 1000), (64, 128, 384), (65, 264, 512),
         (100, 2048, 72), (128, 256, 256), (129, 136, 200), (200, 768, 2056), (256, 64, 1024), (300, 520, 648), (513, 256, 136), (1000, 384, 512)]


@pytest.mark.parametrize("M,D,F", SIZES)
def test_forward(M, D, F):
    check_forward(M, D, F, ("silu", "gelu_tanh", "gelu")[M % 3], False)


@pytest.mark.parametrize("M,D,F", SIZES[::2])
def test_training_forward(M, D, F):
    check_forward(M, D, F, ("silu", "gelu_tanh", "gelu")[(M + 1) % 3], True, scale=3.0)


@pytest.mark.parametrize("M,D,F", SIZES)
def test_backward(M, D, F):
    check_backward(M, D, F, ("silu", "gelu_tanh", "gelu")[M % 3])


def test_many_tiles():
    """Several tiles for every block of the persistent launches, in each product."""
    check_forward(5000, 72, 2600, "silu", True)
    check_backward(5000, 1032, 1544, "gelu_tanh")
    check_forward(100, 1032, 40000, "silu", False)


@pytest.mark.parametrize("M,D,F", [(4100, 64, 72), (700, 136, 2056), (2500, 264, 520), (520, 64, 8200)])
def test_parts_of_k(M, D, F):
    """Few tiles and a long K: the sums of its parts, joined in a second launch, in each product that has such a K."""
    check_forward(M, D, F, "silu", False)
    check_backward(M, D, F, "gelu")


def test_far_rows():
    """Hidden activations beyond 2^31 elements: the last tokens against the formula, and a batch of them alone."""
    M, D, F = 70000, 8, 31000
    X, Wg, Wu, Wd, dout = inputs(M, D, F)
    ffn = B.GatedFFN(FFNConfig(D, F))
    out, dX = torch.empty_like(X), torch.empty_like(X)
    gate, up = (torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ffn.forward(X, Wg, Wu, Wd, out, gate, up)
    last = slice(M - 300, M)
    want = forward_bounds("silu", X[last], Wg, Wu, Wd)
    within(out[last], *want[0], "out")
    within(gate[last], *want[1], "gate")
    within(up[last], *want[2], "up")
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX)
    few, g, u = torch.empty_like(X[last]), gate[last].clone(), up[last].clone()
    ffn.backward(X[last], Wg, Wu, Wd, g, u, dout[last], few)
    # (the same sums in parts of K or in one: fp32 sums of 2 F products each, rounded to bf16)
    within(dX[last], few.double(), 2 * STEP * few.double().abs() + 1e-2, "dX")


def test_shapes_and_empty():
    X, Wg, Wu, Wd, dout = inputs(24, 64, 128)
    ffn = B.GatedFFN(FFNConfig(64, 128))
    flat, deep = torch.empty_like(X), torch.empty_like(X)
    ffn.forward(X, Wg, Wu, Wd, flat)
    ffn.forward(X.view(2, 3, 4, 64), Wg, Wu, Wd, deep.view(2, 3, 4, 64))
    assert torch.equal(flat, deep)
    none = X[:0]
    ffn.forward(none, Wg, Wu, Wd, none)
    h = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda")
    grads = [torch.full_like(w, 7.0) for w in (Wg, Wu, Wd)]
    ffn.backward(none, Wg, Wu, Wd, h, h, none, none, *grads)
    assert not any(g.any() for g in grads)


def test_chosen_gradients():
    """Any subset of the gradients gives the bits of all of them, and the same call the same bits."""
    M, D, F = 300, 136, 264
    X, Wg, Wu, Wd, dout = inputs(M, D, F)
    gate, up = X @ Wg, X @ Wu
    ffn = B.GatedFFN(FFNConfig(D, F))
    like = (X, Wg, Wu, Wd)
    want = [torch.empty_like(t) for t in like]
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, *want)
    for chosen in ((0,), (1, 2), (3,), (0, 3), (0, 1, 2, 3), ()):
        got = [torch.empty_like(t) if i in chosen else None for i, t in enumerate(like)]
        ffn.backward(X, Wg, Wu, Wd, gate, up, dout, *got)
        assert all(torch.equal(got[i], want[i]) for i in chosen)


@pytest.mark.parametrize("M", (5, 300))
def test_special_values(M):
    """A token's infinities and NaN stay its own; gates far out saturate."""
    D, F = 64, 192
    X, Wg, Wu, Wd, _ = inputs(M, D, F)
    ffn = B.GatedFFN(FFNConfig(D, F))
    a, b = torch.empty_like(X), torch.empty_like(X)
    ffn.forward(X, Wg, Wu, Wd, a)
    bad = X.clone()
    bad[1, 3], bad[M - 1, 5] = math.nan, math.inf
    ffn.forward(bad, Wg, Wu, Wd, b)
    rows = torch.ones(M, dtype=torch.bool, device="cuda")
    rows[1] = rows[M - 1] = False
    assert torch.equal(a[rows], b[rows]) and b[1].isnan().all() and not b[M - 1].isfinite().any()
    for activation in ("silu", "gelu_tanh", "gelu"):         # |gate| up to about 1e5: the activation is 0 or the gate
        one = B.GatedFFN(FFNConfig(D, F, activation))
        far = (X.float() * 1e4).to(torch.bfloat16)
        one.forward(far, Wg, Wu, Wd, b)
        want = forward_bounds(activation, far, Wg, Wu, Wd)[0]
        within(b, *want, activation)
        gate, up = far @ Wg, far @ Wu
        grads = [torch.empty_like(t) for t in (X, Wg, Wu, Wd)]
        one.backward(far, Wg, Wu, Wd, gate, up, X, *grads)
        assert all(g.isfinite().all() for g in grads)


@pytest.mark.parametrize("activation", ("silu", "gelu_tanh", "gelu"))
def test_nan_in_the_hidden_activations(activation):
    """A NaN among the kept activations reaches its token's dX and its hidden unit's weights, and nothing else."""
    M, D, F = 140, 72, 200
    X, Wg, Wu, Wd, dout = inputs(M, D, F)
    gate, up = X @ Wg, X @ Wu
    ffn = B.GatedFFN(FFNConfig(D, F, activation))
    clean, got = ([torch.empty_like(t) for t in (X, Wg, Wu, Wd)] for _ in range(2))
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, *clean)
    gate[131, 77] = math.nan
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, *got)
    for a, b, (axis, at) in zip(clean, got, ((0, 131), (1, 77), (1, 77), (0, 77))):
        assert b.select(axis, at).isnan().all()
        keep = torch.ones(b.shape[axis], dtype=torch.bool, device="cuda")
        keep[at] = False
        keep = keep.nonzero().flatten()
        assert torch.equal(a.index_select(axis, keep), b.index_select(axis, keep))


def test_gradient_against_differences():
    """The four gradients against central differences of the formula in 64 bits along random directions: the difference of the
    formula is exact to h^2, and a gradient's own error along a direction is below its bound of test_backward; 2 % of the
    directional derivative's scale covers both at these sizes (2^-8 from each of two roundings, of terms with random signs)."""
    M, D, F = 40, 64, 96
    X, Wg, Wu, Wd, dout = inputs(M, D, F, seed=4)
    for activation in ("silu", "gelu_tanh", "gelu"):
        ffn = B.GatedFFN(FFNConfig(D, F, activation))
        out, gate, up = torch.empty_like(X), *(torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ffn.forward(X, Wg, Wu, Wd, out, gate, up)
        grads = [torch.empty_like(t) for t in (X, Wg, Wu, Wd)]
        ffn.backward(X, Wg, Wu, Wd, gate, up, dout, *grads)
        args = [t.double() for t in (X, Wg, Wu, Wd)]

        def loss(x, wg, wu, wd):
            return ((act(activation, x @ wg) * (x @ wu)) @ wd * dout.double()).sum().item()
        gen = torch.Generator("cuda").manual_seed(6)
        for i, g in enumerate(grads):
            v = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
            v *= args[i].abs().mean()
            e = 1e-5
            plus, minus = ([a + s * e * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
            slope = (loss(*plus) - loss(*minus)) / (2 * e)
            scale = (g.double().norm() * v.norm()).item() / math.sqrt(v.numel())
            assert abs(slope - (g.double() * v).sum().item()) <= 0.02 * scale, (activation, i)


@pytest.mark.parametrize("M", (3, 700))
def test_streams_and_graphs(M):
    """Calls on two streams at once and two captured graphs give what a call alone gives; a graph takes new inputs."""
    D, F = 256, 520
    ffn = B.GatedFFN(FFNConfig(D, F))
    sets = []
    for seed in range(2):
        X, Wg, Wu, Wd, dout = inputs(M, D, F, seed)
        hid = [torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        sets.append((X, Wg, Wu, Wd, dout, hid, [torch.empty_like(t) for t in (X, X, Wg, Wu, Wd)]))

    def call(s):
        X, Wg, Wu, Wd, dout, hid, r = s
        ffn.forward(X, Wg, Wu, Wd, r[0], *hid)
        ffn.backward(X, Wg, Wu, Wd, *hid, dout, *r[1:])

    def same(s, want):
        return all(torch.equal(a, b) for a, b in zip(s[6], want))
    want = []
    for s in sets:
        call(s)
        want.append([t.clone() for t in s[6]])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                call(s)
    torch.cuda.synchronize()
    assert all(same(s, w) for s, w in zip(sets, want))
    graphs = []
    for s in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(s)
        graphs.append(graph)
    for s in sets:
        for t in s[6]:
            t.zero_()
    torch.cuda.synchronize()
    for _ in range(3):
        for graph, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    assert all(same(s, w) for s, w in zip(sets, want))
    for a, b in zip(sets[0][:5], sets[1][:5]):
        a.copy_(b)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert same(sets[0], want[1]) and ffn.device_status() == 0


def test_binding_refusals():
    X, Wg, Wu, Wd, dout = inputs(4, 64, 128)
    ffn = B.GatedFFN(FFNConfig(64, 128))
    h = torch.empty(4, 128, dtype=torch.bfloat16, device="cuda")
    y = torch.empty_like(X)
    for call in (lambda: ffn.forward(X.float(), Wg, Wu, Wd, y), lambda: ffn.forward(X, Wg.t(), Wu, Wd, y), lambda: ffn.forward(X, Wg, Wu, Wg, y),
                 lambda: ffn.forward(X, Wg, Wu, Wd, y[:3]), lambda: ffn.forward(X, Wg, Wu, Wd, y, gate=h), lambda: ffn.forward(X.cpu(), Wg, Wu, Wd, y),
                 lambda: ffn.forward(X[:, :32], Wg, Wu, Wd, y), lambda: ffn.forward(X, Wg, Wu, Wd.t().contiguous().t(), y),
                 lambda: ffn.forward(X.flatten()[1:193].view(3, 64), Wg, Wu, Wd, y[:3]),
                 lambda: ffn.backward(X, Wg, Wu, Wd, h, h, dout, dWg=torch.empty_like(Wg)), lambda: ffn.backward(X, Wg, Wu, Wd, h, h[:2], dout),
                 lambda: B.GatedFFN(FFNConfig(60, 128)), lambda: B.GatedFFN(FFNConfig(64, 128, "relu"))):
        with pytest.raises(B.FFError):
            call()


def test_overlap():
    """What a launch would read while it is written is refused; what has been read by then may be written over."""
    M, D, F = 40, 128, 128                       # (one size for all: any tensor may be laid over any other)
    X, Wg, Wu, Wd, dout = inputs(M, D, F)
    gate, up = X @ Wg, X @ Wu
    ffn = B.GatedFFN(FFNConfig(D, F))
    out, dX, y = (torch.empty_like(X) for _ in range(3))
    grads = [torch.empty_like(t) for t in (Wg, Wu, Wd)]
    ffn.forward(X, Wg, Wu, Wd, out)
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX, *grads)

    def refused(call):
        with pytest.raises(B.FFError) as e:
            call()
        assert e.value.status == 1 and "overlap" in str(e.value)
    both = torch.cat([X, X])                     # rows 0 .. M-1 and 1 .. M of it overlap
    part, shifted = both[:M], both[1:M + 1]
    refused(lambda: ffn.forward(X, Wg, Wu, Wd, y, X, up))
    refused(lambda: ffn.forward(X, Wg, Wu, Wd, y, gate, gate))
    refused(lambda: ffn.forward(X, Wg, Wu, Wd, gate, gate, up))
    refused(lambda: ffn.forward(X, Wg, Wu, Wd, y, Wd[:M], up))
    refused(lambda: ffn.forward(X, Wg, Wu, Wd, Wd[:M]))
    refused(lambda: ffn.forward(part, Wg, Wu, Wd, y, shifted, up))
    for bad in (X, dout, Wg[:M], Wu[:M], grads[2][:M]):
        refused(lambda: ffn.backward(X, Wg, Wu, Wd, gate, up, dout, bad, *grads))
    refused(lambda: ffn.backward(part, Wg, Wu, Wd, gate, up, dout, shifted, *grads))
    refused(lambda: ffn.backward(X, Wg, Wu, Wd, gate, up, dout, None, grads[0], grads[0]))
    refused(lambda: ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX, Wg, grads[1]))
    lib, need = B.library(), C.c_size_t()
    args = [t.data_ptr() for t in (X, Wg, Wu, Wd)]
    B._check(lib.ff_ffn_workspace_bytes(C.byref(ffn._c), M, False, C.byref(need)))
    store = torch.empty(need.value + 2 * X.numel(), dtype=torch.uint8, device="cuda")
    over = store[need.value - 256:].data_ptr()   # its first 256 bytes are the workspace's last
    assert lib.ff_ffn_forward(ffn.handle, M, *args, None, None, over, store.data_ptr(), need.value, None) == 1
    # what has been read: out over X, dX over gate, dWd over Wd, dX over dout without dWd, over X without dWg
    z = X.clone()
    ffn.forward(z, Wg, Wu, Wd, z)
    assert torch.equal(z, out)
    g, w, u = gate.clone(), Wd.clone(), up.clone()
    ffn.backward(X, Wg, Wu, w, g, u, dout, g, grads[0], u.new_empty(D, F), w)
    assert torch.equal(g, dX) and torch.equal(w, grads[2])
    z = dout.clone()
    ffn.backward(X, Wg, Wu, Wd, gate, up, z, z)
    assert torch.equal(z, dX)
    z = X.clone()
    ffn.backward(z, Wg, Wu, Wd, gate, up, dout, z, dWd=grads[2])
    assert torch.equal(z, dX)


def test_status_of_a_new_handle():
    """A handle's status word is clear for every stream from the start, also where the default stream is busy while it is made and the
    word's memory held something else before."""
    runtime = C.CDLL("libcudart.so.12")
    blocks = [C.c_void_p() for _ in range(64)]
    for b in blocks:
        assert runtime.cudaMalloc(C.byref(b), C.c_size_t(256)) == 0
        assert runtime.cudaMemset(b, 255, C.c_size_t(256)) == 0
    torch.cuda.synchronize()
    for b in blocks:
        assert runtime.cudaFree(b) == 0
    side = torch.cuda.Stream()
    torch.cuda._sleep(200_000_000)
    ffn = B.GatedFFN(FFNConfig(64, 128))
    with torch.cuda.stream(side):
        assert ffn.device_status() == 0
    torch.cuda.synchronize()


def exact_inputs(M, D, F, live=None, seed=0):
    """Small whole numbers for which every sum of the block is exact in fp32 and H, dG and dU are exact in bf16, whatever the order of
    the sums: X is 1 in the first column and -1, 0 or 1 elsewhere; a column of Wg is 32 in the first row and has four more ones, one of Wu
    four; so gates are 28 .. 36, where each activation is the gate itself and its slope 1 (e^-28 is below half a step of 1 in fp32), up is
    -4 .. 4 and |H| <= 144.  dout has four ones a row (none but in the last `live` rows): |dH| <= 4 times the columns' chance of meeting."""
    gen = torch.Generator("cuda").manual_seed(seed)

    def three(*shape):
        return torch.randint(-1, 2, shape, generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16)

    def four_ones(rows, cols, first=0):
        """[rows][cols] with +-1 in four random places (or fewer, where two meet) of each row, from column `first` on"""
        t = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
        at = torch.randint(first, cols, (rows, 4), generator=gen, device="cuda")
        return t.scatter_(1, at, (2 * torch.randint(0, 2, (rows, 4), generator=gen, device="cuda") - 1).to(torch.bfloat16))
    X, Wd, dout = three(M, D), three(F, D), four_ones(M, D)
    X[:, 0] = 1
    Wg, Wu = (four_ones(F, D, 1).t().contiguous() for _ in range(2))
    Wg[0] = 32
    if live is not None:
        dout[:M - live] = 0
    return X, Wg, Wu, Wd, dout


def check_exact(M, D, F, activation, rows=None):
    """Every output is the exact number rounded once, bit for bit: no part of a sum is left out or added twice.  With `rows`, what belongs to
    tokens is compared for that many at the end, the only ones with a gradient."""
    X, Wg, Wu, Wd, dout = exact_inputs(M, D, F, rows)
    ffn = B.GatedFFN(FFNConfig(D, F, activation))
    out, dX, gate, up = torch.empty_like(X), torch.empty_like(X), *(torch.empty(M, F, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ffn.forward(X, Wg, Wu, Wd, out, gate, up)
    alone = torch.empty_like(X)
    ffn.forward(X, Wg, Wu, Wd, alone)
    grads = [torch.empty_like(t) for t in (Wg, Wu, Wd)]
    ffn.backward(X, Wg, Wu, Wd, gate, up, dout, dX, *grads)
    assert ffn.device_status() == 0
    end = slice(M - (rows or M), M)
    x, do, wg, wu, wd = (t.double() for t in (X[end], dout[end], Wg, Wu, Wd))
    g, u = x @ wg, x @ wu
    h, dh = g * u, do @ wd.T
    dg, du = dh * u, dh * g
    for t in (g, u, h, dg, du):
        assert torch.equal(t, t.to(torch.bfloat16).double())
    for got, want, name in ((gate[end], g, "gate"), (up[end], u, "up"), (out[end], h @ wd, "out"), (alone[end], h @ wd, "out alone"),
                            (dX[end], dg @ wg.T + du @ wu.T, "dX"), (grads[0], x.T @ dg, "dWg"), (grads[1], x.T @ du, "dWu"), (grads[2], h.T @ do, "dWd")):
        assert want.abs().max() < 2 ** 24, name
        assert torch.equal(got, want.to(torch.bfloat16)), f"{name}: {int((got != want.to(torch.bfloat16)).sum())} of {want.numel()}"


@pytest.mark.parametrize("M,D,F", [(1, 256, 520), (1, 1032, 40000), (13, 2048, 5632), (37, 1032, 4104), (100, 1032, 40000), (300, 520, 648), (513, 256, 136),
                                   (700, 136, 2056), (4100, 64, 72), (5000, 1032, 1544), (20000, 264, 520)])
def test_exact_sums(M, D, F):
    check_exact(M, D, F, ("silu", "gelu_tanh", "gelu")[M % 3])


def test_far_rows_exact():
    """Hidden activations and their gradients beyond 2^31 elements: the last tokens' outputs and all gradients, which only these tokens have."""
    check_exact(70000, 8, 31000, "silu", 300)
