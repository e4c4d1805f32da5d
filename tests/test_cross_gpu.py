"""Cross attention against its formulas in 64 bits.

Tolerances, element by element.  A score is a sum of d products in fp32, d 2^-22 of the sum of their sizes off (2^-23 for every addition,
whichever way the tensor core cuts), times the scale; in units of log2, with the maximum taken away, its size costs another
4 x 2^-24; the exponential is 2^-21 off.  So an unnormalised probability is off by e = that, relatively, and by 2^-8 more where it is
rounded to bf16 for a product.  Sums of K terms in fp32 add K 2^-22 of the sum of their sizes; results are rounded to bf16: 2^-8."""
import ctypes as C
import math

import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import CrossAttentionConfig

pytestmark = pytest.mark.gpu
STEP = 2.0 ** -8
NAN = float("nan")


def summed(n):
    return n * 2.0 ** -22


def within(got, want, bound, what):
    over = (got.double() - want).abs() - bound
    assert not torch.isnan(over).any(), what
    assert over.max().item() <= 0, f"{what}: {over.max().item():.3g} beyond the bound at {int(over.argmax())}"


class Case:
    """Inputs of one call, in tensors whose surroundings are watched, and what the formulas make of them."""

    def __init__(self, B_, N, K, H, G, d, order="tokens_first", keys="all", scale=0.0, spoil=True, seed=0, size=1.5):
        self.shape, self.H, self.G, self.d = (B_, N, K), H, G, d
        gen = torch.Generator("cuda").manual_seed(seed + 1000 * N + K)

        def rows(heads, tokens, s=1.0):
            return (s * torch.randn(B_, heads, tokens, d, generator=gen, device="cuda")).to(torch.bfloat16)
        self.q, self.k, self.v, self.dout = (self.place(t, order) for t in (rows(H, N, size), rows(G, K), rows(G, K), rows(H, N)))
        self.lengths = self.mask = None
        counts = torch.ones(B_, K, dtype=torch.bool, device="cuda")
        if keys in ("lengths", "both"):
            values = [K, 0, max(1, K // 3), K + 9, -5, K - 1][:B_] if B_ > 1 else [max(1, K - 3)]
            self.lengths = torch.tensor((values * B_)[:B_], dtype=torch.int32, device="cuda")
            counts &= torch.arange(K, device="cuda") < self.lengths[:, None]
        if keys in ("mask", "both"):
            self.mask = torch.rand(B_, K, generator=gen, device="cuda") < 0.6
            if B_ > 2:
                self.mask[2] = False
            counts &= self.mask
        self.counts = counts
        if spoil and keys != "all":                           # rows that do not count hold anything
            gone = ~counts[:, None, :, None].expand(B_, G, K, d)
            self.k[gone], self.v[gone] = NAN, float("inf")
        self.order = order
        self.scale = scale if scale else d ** -0.5
        self.attention = B.CrossAttention(CrossAttentionConfig(d, H, G, scale))

    @staticmethod
    def place(t, order):
        """The same values, head by head or token by token, or in rows of a wider tensor."""
        if order == "heads_first":
            return t.contiguous()
        if order == "tokens_first":
            return t.transpose(1, 2).contiguous().transpose(1, 2)
        b, h, n, d = t.shape
        wide = torch.full((b, n + 2, h + 1, d + 16), NAN, dtype=t.dtype, device="cuda")
        view = wide[:, 1:n + 1, :h, 8:d + 8].transpose(1, 2)
        view.copy_(t)
        return view

    def empty(self, like):
        """A result's place, NaN, and a function that says whether nothing around it was touched."""
        b, h, n, d = like.shape
        if self.order == "heads_first":
            store = torch.full((b, h, n + 3, d + 8), NAN, dtype=torch.bfloat16, device="cuda")
            view = store[:, :, :n, :d]
        else:
            store = torch.full((b, n + 3, h + 1, d + 8), NAN, dtype=torch.bfloat16, device="cuda")
            view = store[:, :n, :h, :d].transpose(1, 2)

        def clean():
            view.fill_(NAN)
            return bool(store.isnan().all())
        return view, clean

    def reference(self, lse=None, out=None):
        """Results and bounds; with lse and out (what the forward call left) those of the gradients too."""
        B_, N, K = self.shape
        H, G, d, grp = self.H, self.G, self.d, self.H // self.G
        gone = ~self.counts[:, None, None, :]
        k, v = (t.double().masked_fill(gone.transpose(-1, -2), 0).repeat_interleave(grp, 1) for t in (self.k, self.v))
        q = self.q.double()
        s = (q @ k.transpose(-1, -2)) * self.scale
        es = summed(d) * (q.abs() @ k.abs().transpose(-1, -2)) * self.scale
        some = self.counts.any(-1)[:, None, None]
        top = s.masked_fill(gone, -math.inf).amax(-1, keepdim=True).masked_fill(~some[..., None], 0)
        p = (s - top).exp().masked_fill(gone, 0)
        e = es + 2.0 ** -22 * (s.abs() + top.abs()) + 2.0 ** -21
        total = p.sum(-1, keepdim=True).clamp_min(1e-300)
        p = p / total
        ebar = (p * e).sum(-1, keepdim=True) + summed(K)
        o = p @ v
        size = p @ v.abs()
        eo = (p * (e + STEP)) @ v.abs() + (ebar + summed(K)) * size
        eo = STEP * o.abs() + (1 + STEP) * eo * 1.01
        L = (top + total.log())[..., 0].masked_fill(~some, -math.inf)
        eL = ebar[..., 0] + 2.0 ** -21 * (1 + top[..., 0].abs() + L.abs().masked_fill(~some, 0))
        res = {"out": (o, eo), "lse": (L, eL)}
        if lse is None:
            return res
        do = self.dout.double()
        P = p
        eP = e + eL[..., None] + 2.0 ** -22 * L.abs().masked_fill(~some, 0)[..., None]
        dP = do @ v.transpose(-1, -2)
        D = (P * dP).sum(-1, keepdim=True)
        eD = (do.abs() * eo).sum(-1, keepdim=True) + summed(d) * (do.abs() * (o.abs() + eo)).sum(-1, keepdim=True)
        edP = summed(d) * (do.abs() @ v.abs().transpose(-1, -2))
        dS = P * (dP - D)
        edS = P * (1 + eP) * (edP + eD + 2.0 ** -23 * (dP.abs() + D.abs())) + dS.abs() * (eP + STEP) * 1.01

        def per_key_head(t):
            return t.view(B_, G, grp, K, d).sum(2)
        dq = self.scale * (dS @ k)
        edq = self.scale * (edS @ k.abs() + summed(K) * ((dS.abs() + edS) @ k.abs()))
        res["dq"] = dq, STEP * dq.abs() + (1 + STEP) * edq
        n = summed(N * grp)
        dk = per_key_head(self.scale * (dS.transpose(-1, -2) @ q))
        edk = per_key_head(self.scale * ((edS + n * (dS.abs() + edS)).transpose(-1, -2) @ q.abs()))
        res["dk"] = dk, STEP * dk.abs() + (1 + STEP) * edk
        dv = per_key_head(P.transpose(-1, -2) @ do)
        edv = per_key_head((P * (eP + STEP) * 1.01 + n * P).transpose(-1, -2) @ do.abs())
        res["dv"] = dv, STEP * dv.abs() + (1 + STEP) * edv
        return res

    def check(self, backward=True):
        B_, N, K = self.shape
        out, out_clean = self.empty(self.q)
        lse = torch.full((B_, self.H, N), NAN, device="cuda")
        self.attention.forward(self.q, self.k, self.v, out, lse, self.lengths, self.mask)
        want = self.reference(lse, out)
        within(out, *want["out"], "out")
        value, bound = want["lse"]
        none = value == -math.inf
        assert torch.equal(lse == -math.inf, none)
        within(lse.masked_fill(none, 0), value.masked_fill(none, 0), bound, "lse")
        again = torch.empty_like(out)
        self.attention.forward(self.q, self.k, self.v, again, None, self.lengths, self.mask)
        assert torch.equal(again, out)
        if backward:
            (dq, dq_clean), (dk, dk_clean), (dv, dv_clean) = self.empty(self.q), self.empty(self.k), self.empty(self.v)
            args = (self.q, self.k, self.v, out, lse, self.dout)
            keys = {"lengths": self.lengths, "mask": self.mask}
            self.attention.backward(*args, dq, dk, dv, **keys)
            for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
                within(got, *want[name], name)
            gone = ~self.counts[:, None, :, None].expand_as(dk)
            assert (dk[gone] == 0).all() and (dv[gone] == 0).all()
            # one without the other: the same bits
            dq2, dk2, dv2 = torch.empty_like(dq), torch.empty_like(dk), torch.empty_like(dv)
            self.attention.backward(*args, dq2, **keys)
            self.attention.backward(*args, None, dk2, dv2, **keys)
            assert torch.equal(dq2, dq)
            for name, got in (("dk", dk2), ("dv", dv2)):     # (D of its own launch is summed in another order)
                within(got, *want[name], name)
            again = [torch.empty_like(t) for t in (dq, dk, dv)]
            self.attention.backward(*args, *again, **keys)
            assert all(torch.equal(a, b) for a, b in zip(again, (dq, dk, dv)))
            assert dq_clean() and dk_clean() and dv_clean()
        assert self.attention.device_status() == 0
        assert out_clean()


@pytest.mark.parametrize("N", [1, 37, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("K", [1, 5, 127, 128, 129, 385])
def test_lengths(N, K):
    Case(2, N, K, 4, 2, 64).check()
    Case(1, N, K, 2, 2, 128, "heads_first").check()


@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 120, 128])
@pytest.mark.parametrize("order", ["heads_first", "tokens_first", "wide"])
def test_head_dims_and_strides(d, order):
    Case(2, 140, 150, 4, 2, d, order).check()
    Case(2, 3, 150, 4, 1, d, order, "mask").check()


@pytest.mark.parametrize("keys", ["lengths", "mask", "both"])
@pytest.mark.parametrize("shape", [(6, 70, 300, 4, 4, 64), (6, 130, 131, 6, 2, 128), (3, 1, 260, 8, 2, 128), (4, 9, 700, 4, 2, 32), (3, 260, 77, 2, 1, 80)])
def test_keys_that_do_not_count(keys, shape):
    Case(*shape, keys=keys).check()


@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (12, 4), (7, 1), (16, 2), (40, 8)])
@pytest.mark.parametrize("N", [1, 20, 33, 150])
def test_shared_key_heads(heads, N):
    Case(2, N, 200, *heads, 64, keys="lengths").check()


@pytest.mark.parametrize("shape", [(1, 1, 9000, 4, 2, 128), (2, 5, 5000, 2, 2, 64), (1, 200, 3333, 2, 1, 96), (1, 3000, 200, 2, 2, 128), (2, 2500, 140, 6, 2, 64),
                                   (8, 1, 1200, 8, 2, 128)])
def test_keys_and_queries_in_parts(shape):
    """Few tiles: the keys (backward the queries too) are cut, and the parts joined; samples whose parts are empty among them."""
    Case(*shape).check()
    Case(*shape, keys="lengths").check()


def test_scale_and_large_scores():
    Case(1, 100, 140, 2, 2, 64, scale=0.5).check()
    Case(1, 100, 600, 2, 2, 64, size=200.0).check(backward=False)       # the maximum grows from tile to tile
    c = Case(1, 130, 512, 1, 1, 64, size=20.0)
    c.k.mul_(torch.linspace(0.1, 4, 512, device="cuda")[:, None].to(torch.bfloat16))
    c.check(backward=False)


def test_very_low_scores():
    """A row whose scores all lie below -1e30, or are equal and large, is a softmax like any other."""
    c = Case(1, 64, 200, 1, 1, 64)
    c.q.fill_(2.0 ** 54), c.k.fill_(-2.0 ** 54)
    out, lse = torch.empty_like(c.q), torch.empty(1, 1, 64, device="cuda")
    c.attention.forward(c.q, c.k, c.v, out, lse)
    mean = c.v.double().mean(2, keepdim=True)
    within(out, mean.expand_as(out), STEP * mean.abs() + 2.0 ** -7 * c.v.double().abs().mean(2, keepdim=True), "mean")
    assert (lse < -1e30).all() and lse.isfinite().all()


@pytest.mark.parametrize("value", [NAN, float("inf")])
def test_a_query_that_is_not_finite_spoils_itself_alone(value):
    c = Case(2, 150, 140, 2, 2, 64)
    clean, out = torch.empty_like(c.q), torch.empty_like(c.q)
    c.attention.forward(c.q, c.k, c.v, clean)
    c.q[1, 0, 77, 5] = value
    c.attention.forward(c.q, c.k, c.v, out)
    assert out[1, 0, 77].isnan().all()
    out[1, 0, 77] = clean[1, 0, 77]
    assert torch.equal(out, clean)


def test_a_value_that_is_not_finite_reaches_who_counts_it():
    c = Case(2, 150, 300, 2, 1, 64, keys="mask", spoil=False)
    c.mask[:] = True
    c.mask[0, 130] = False
    c.v[:, 0, 130, 7] = NAN
    out = torch.empty_like(c.q)
    c.attention.forward(c.q, c.k, c.v, out, mask=c.mask)
    assert out[0].isfinite().all() and out[1, :, :, 7].isnan().all()


def test_shared_states_and_output_over_input():
    """States of stride zero in the batch (the same for all samples) or the heads; out in the place of q."""
    c = Case(3, 150, 200, 4, 4, 64)
    k, v = c.k[:1].expand(3, -1, -1, -1), c.v[:, :1].expand(-1, 4, -1, -1)
    out, want = torch.empty_like(c.q), torch.empty_like(c.q)
    c.attention.forward(c.q, k, v, out)
    c.attention.forward(c.q, k.contiguous(), v.contiguous(), want)
    assert torch.equal(out, want)
    for N, K in ((150, 200), (1, 5000)):
        c = Case(1, N, K, 4, 2, 128)
        want = torch.empty_like(c.q)
        c.attention.forward(c.q, c.k, c.v, want)
        c.attention.forward(c.q, c.k, c.v, c.q)
        assert torch.equal(c.q, want)


def test_no_rows():
    for B_, N, K in ((0, 5, 5), (2, 0, 5), (2, 5, 0), (2, 200, 0), (3, 0, 0)):
        a = B.CrossAttention(CrossAttentionConfig(64, 4, 2))
        q, k = torch.full((B_, 4, N, 64), 1.0, dtype=torch.bfloat16, device="cuda"), torch.full((B_, 2, K, 64), 1.0, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.full_like(q, NAN), torch.full((B_, 4, N), NAN, device="cuda")
        a.forward(q, k, k, out, lse)
        assert (out == 0).all() and (lse == -math.inf).all()
        dq, dk, dv = torch.full_like(q, NAN), torch.full_like(k, NAN), torch.full_like(k, NAN)
        a.backward(q, k, k, out, lse, q, dq, dk, dv)
        assert (dq == 0).all() and (dk == 0).all() and (dv == 0).all() and a.device_status() == 0


def test_gradient_against_differences():
    """A step of a whole tensor along a direction against the gradient's product with it."""
    c = Case(2, 40, 50, 4, 2, 32, keys="mask", spoil=False)

    def loss(q, k, v):
        o = c.reference.__func__(_with(c, q, k, v))["out"][0]
        return (o * c.dout.double()).sum().item()

    def _with(c, q, k, v):
        o = object.__new__(Case)
        o.__dict__.update(c.__dict__)
        o.q, o.k, o.v = q, k, v
        return o
    out, lse = torch.empty_like(c.q), torch.empty(2, 4, 40, device="cuda")
    c.attention.forward(c.q, c.k, c.v, out, lse, mask=c.mask)
    grads = [torch.empty_like(t) for t in (c.q, c.k, c.v)]
    c.attention.backward(c.q, c.k, c.v, out, lse, c.dout, *grads, mask=c.mask)
    leaves = [t.double() for t in (c.q, c.k, c.v)]
    bounds = c.reference(lse, out)
    for i, name in enumerate(("dq", "dk", "dv")):
        way = torch.randn(leaves[i].shape, generator=torch.Generator("cuda").manual_seed(i), device="cuda", dtype=torch.float64)
        h = 1e-4
        ends = [loss(*[t + (s * h * way if j == i else 0) for j, t in enumerate(leaves)]) for s in (1, -1)]
        slope, got = (ends[0] - ends[1]) / (2 * h), (grads[i].double() * way).sum().item()
        assert abs(slope - got) <= (bounds[name][1] * way.abs()).sum().item() + 1e-5 * abs(slope) + 1e-4


def test_offsets_beyond_two_to_the_31():
    """A cache whose last sample lies 2^32 bytes and more behind the first."""
    K, G, d = 70000, 8, 128
    k = torch.empty(32, G, K, d, dtype=torch.bfloat16, device="cuda")
    small = Case(1, 3, K, 16, G, d, "heads_first")
    k[0], k[31] = small.k[0], small.k[0]
    a, out, want = small.attention, torch.empty(32, 16, 3, d, dtype=torch.bfloat16, device="cuda"), torch.empty_like(small.q)
    lengths = torch.zeros(32, dtype=torch.int32, device="cuda")
    lengths[31] = lengths[0] = K
    q = small.q.expand(32, -1, -1, -1).contiguous()
    a.forward(q, k, k, out, lengths=lengths)
    a.forward(small.q, small.k, small.k, want)
    small.v = small.k
    within(out[31:], *small.reference()["out"], "out")
    assert torch.equal(out[0], out[31]) and (out[1:31] == 0).all()


def test_streams_and_graphs():
    """Captured calls that share a handle, and calls on another stream than the tensors were made on."""
    cases = [Case(1, 1, 5000, 8, 2, 64, seed=s) for s in range(2)] + [Case(2, 300, 180, 4, 2, 128, keys="lengths")]
    handles = {}
    calls = []
    for c in cases:
        a = handles.setdefault((c.H, c.G, c.d), c.attention)
        out, lse = torch.empty_like(c.q), torch.empty(c.shape[0], c.H, c.shape[1], device="cuda")
        grads = [torch.empty_like(t) for t in (c.q, c.k, c.v)]
        kw = {"lengths": c.lengths, "mask": c.mask}
        calls.append((a, (c.q, c.k, c.v), out, lse, c.dout, grads, kw))

    def run():
        for a, x, out, lse, dout, grads, kw in calls:
            a.forward(*x, out, lse, **kw)
            a.backward(*x, out, lse, dout, *grads, **kw)
    results = [t for c in calls for t in (c[2], c[3], *c[5])]
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in results]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for again in (graph.replay, graph.replay):
        for t in results:
            t.fill_(NAN)
        again()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in results:
            t.fill_(NAN)
        run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    assert all(c[0].device_status() == 0 for c in calls)


def test_refused_calls():
    """Refused before anything runs, with a message of the handle."""
    lib, a = B.library(), B.CrossAttention(CrossAttentionConfig(64, 4, 2))
    t = torch.zeros(1 << 16, dtype=torch.bfloat16, device="cuda")
    p = t.data_ptr()

    def heads(data=p, sb=2560, sh=640, st=64, n=4):
        return C.byref(B.ff_heads_t(data, sb, sh, st, n))
    kv = heads(p + 20480, 1280, 640, 64, 2)

    def forward(batch=2, queries=10, keys=10, q=heads(), k=kv, v=kv, lengths=None, mask=None, out=heads(p + 40960), lse=None, ws=None, n=0):
        return lib.ff_cross_attention_forward(a.handle, batch, queries, keys, q, k, v, lengths, mask, out, lse, ws, n, None)

    def backward(q=heads(), k=kv, v=kv, out=heads(p + 40960), lse=p + 65536, dout=heads(p + 40960), dq=heads(p + 81920), dk=heads(p + 61440, 1280, 640, 64, 2),
                 dv=heads(p + 66560, 1280, 640, 64, 2), ws=p + 102400 // 256 * 256, n=1 << 14):
        return lib.ff_cross_attention_backward(a.handle, 2, 10, 10, q, k, v, None, None, out, lse, dout, dq, dk, dv, ws, n, None)
    assert forward() == 0
    for kw in ({"batch": -1}, {"queries": -1}, {"keys": -1}, {"q": None}, {"out": None}, {"k": None}, {"q": heads(0)}, {"q": heads(n=2)}, {"k": heads(n=4)},
               {"q": heads(sb=-64)}, {"out": heads(st=0)}, {"out": heads(sh=0)}, {"out": heads(sb=0)}, {"lse": p + 2}, {"lengths": p + 1}):
        assert forward(**kw) == 1, kw
        assert lib.ff_cross_attention_last_error(a.handle)
    for kw in ({"queries": 1 << 31}, {"keys": 1 << 31}, {"batch": 1 << 30}, {"q": heads(p + 2)}, {"q": heads(sb=2561)}, {"out": heads(sh=644)}, {"k": heads(st=68, n=2)},
               {"q": heads(st=0)}, {"q": heads(sh=0)}, {"k": heads(st=0, n=2)}, {"v": heads(sb=1 << 40, n=2)}):
        assert forward(**kw) == 2, kw
    assert forward(queries=1, keys=5000, batch=1) == 3
    for kw in ({"dk": None}, {"dv": None}, {"lse": None}, {"dout": None}, {"dq": heads()}, {"dq": heads(p + 40960)}, {"dk": kv}, {"dv": heads(p + 61440, 1280, 640, 64, 2)},
               {"dq": heads(p + 81920, st=0)}):
        assert backward(**kw) == 1, kw
    assert backward(ws=None) == 3 and backward(n=8) == 3 and backward(ws=p + 16) == 3
    torch.cuda.synchronize()
    assert a.device_status() == 0
