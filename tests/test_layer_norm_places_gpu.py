"""Layer norm of rows at every alignment: lengths that would move in pieces of 16 bytes at addresses, or with strides, that do not allow it, tensors of
one call aligned differently from one another, and offsets beyond 2^31 elements.  The values are those of aligned tensors: y and dx within one rounding
of each other (another piece sums in another order), the weights' gradients within the bounds of their sums."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import LayerNormConfig
from test_layer_norm_gpu import TYPE, normal, reference, within, HALF

pytestmark = pytest.mark.gpu


def place(t, start, token=0):
    """The same values, `start` elements into a tensor whose rows lie `token` elements further apart; the tensor around them."""
    b, n, d = t.shape
    store = torch.full((start + b * n * (d + token) + 16,), float("nan"), dtype=t.dtype, device="cuda")
    view = store.as_strided((b, n, d), (n * (d + token), d + token, 1), start)
    view.copy_(t)
    return store, view


def check(dtype, shape, starts, tokens=(0, 0, 0, 0), per_sample=False):
    """x, dy, y and dx at the given starts and distances of rows."""
    d, half = shape[-1], HALF[dtype]
    x, dy = normal(*shape, seed=1).to(TYPE[dtype]), normal(*shape, seed=2).to(TYPE[dtype])
    wshape = (shape[0], d) if per_sample else (d,)
    w, b = normal(*wshape, seed=3, mean=1.0), normal(*wshape, seed=4)
    nan = torch.full_like(x, float("nan"))
    (_, xv), (_, gv), (ys, yv), (ds, dv) = (place(t, s, k) for t, s, k in zip((x, dy, nan, nan), starts, tokens))
    norm = B.LayerNorm(LayerNormConfig(d, dtype, 1e-5))
    dw, db = torch.full_like(w, float("nan")), torch.full_like(w, float("nan"))
    norm.forward(xv, w, b, yv)
    norm.backward(xv, w, gv, dv, dw, db)
    want = reference(x, w, b, dy, 0.0, per_sample)
    for got, name in ((yv, "y"), (dv, "dx")):
        value, e = want[name]
        within(got, value, half * value.abs() + (1 + half) * e, name)
    within(dw, *want["dw"], "dweight"), within(db, *want["db"], "dbias")
    for s, v in ((ys, yv), (ds, dv)):
        v.fill_(float("nan"))
        assert s.isnan().all()


@pytest.mark.parametrize("dtype,start", [("bf16", s) for s in range(1, 8)] + [("fp32", s) for s in range(1, 4)])
@pytest.mark.parametrize("dim", [64, 1024, 2048, 4160])
def test_starts(dtype, start, dim):
    check(dtype, (2, 37, dim), (start,) * 4, per_sample=dim == 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("starts", [(0, 1, 0, 0), (1, 0, 0, 0), (0, 0, 3, 0), (0, 0, 0, 2), (2, 4, 1, 0)])
def test_tensors_aligned_differently(dtype, starts):
    check(dtype, (3, 50, 1024), starts)
    check(dtype, (1, 300, 256), starts, per_sample=True)


@pytest.mark.parametrize("dtype,token", [("bf16", 1), ("bf16", 2), ("bf16", 4), ("fp32", 1), ("fp32", 2)])
def test_rows_at_odd_distances(dtype, token):
    check(dtype, (2, 41, 512), (0,) * 4, (token,) * 4)
    check(dtype, (2, 41, 8192), (0,) * 4, (0, token, 0, 0))


@pytest.mark.parametrize("dtype,dim", [("bf16", 1024), ("bf16", 1001), ("fp32", 260)])
def test_offsets_beyond_two_to_the_31(dtype, dim):
    """Rows 2^26 elements apart and samples 2^31, of all tensors of a call, forward and backward."""
    B_, N, e = 2, 20, TYPE[dtype]
    far, apart = (1 << 31) + 64, (1 << 26) + 8
    pool = torch.empty(far + N * apart + (1 << 16), dtype=e, device="cuda")
    x, dy = normal(B_, N, dim, seed=1).to(e), normal(B_, N, dim, seed=2).to(e)
    w, b = normal(B_, dim, seed=3), normal(B_, dim, seed=4)
    views = [pool.as_strided((B_, N, dim), (far, apart, 1), i * 4096) for i in range(4)]
    views[0].copy_(x), views[1].copy_(dy)
    norm = B.LayerNorm(LayerNormConfig(dim, dtype, 1e-5))
    results = []
    for xv, gv, yv, dv in (views, (x, dy, torch.empty_like(x), torch.empty_like(x))):
        dw, db = torch.empty_like(w), torch.empty_like(w)
        norm.forward(xv, w, b, yv)
        norm.backward(xv, w, gv, dv, dw, db)
        results.append((yv, dv, dw, db))
    assert all(torch.equal(a, c) for a, c in zip(*results))
