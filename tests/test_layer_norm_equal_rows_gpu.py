"""Layer norm of rows whose values are all the same, up to the ends of fp32: their variance is zero, n is zero, y the bias, and they leave the
weights' gradients alone."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import LayerNormConfig

pytestmark = pytest.mark.gpu
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-5


def normal(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


def check(dtype, dim, values, weights):
    """Rows of one value each with rows of many between them."""
    t, n = TYPE[dtype], len(values)
    x, dy = normal(2 * n + 1, dim, seed=dim).to(t), normal(2 * n + 1, dim, seed=dim + 1).to(t)
    x[1::2] = torch.tensor(values, device="cuda", dtype=t)[:, None]
    w, b = (normal(dim, seed=dim + 2), normal(dim, seed=dim + 3)) if weights else (None, None)
    norm = B.LayerNorm(LayerNormConfig(dim, dtype, EPS))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    norm.forward(x, w, b, y)
    norm.backward(x, w, dy, dx, dw, db)
    want = torch.zeros(dim, device="cuda") if b is None else b
    assert torch.equal(y[1::2], want.to(t).expand(n, dim))
    # n = 0: dx = r (g - mean g) with r = eps^-1/2.  The mean's sum runs over fewer than 64 additions one after the other; product, difference,
    # square root and the last product are another eight roundings.
    g = dy[1::2].double() * (1.0 if w is None else w.double())
    wanted = EPS ** -0.5 * (g - g.mean(-1, keepdim=True))
    bound = 72 * 2.0 ** -24 * EPS ** -0.5 * (g.abs() + g.abs().mean(-1, keepdim=True)) + HALF[dtype] * wanted.abs()
    assert ((dx[1::2].double() - wanted).abs() <= bound).all()
    # dweight is that of the other rows, sums of n + 1 terms; n is off by 190 x 2^-24 (|n| + 1) at most (tests/test_layer_norm_means_gpu.py: the mean of
    # 96 values and more lies within half a deviation, that of one or two is a sum of as many)
    X, DY = x[0::2].double(), dy[0::2].double()
    c = X - X.mean(-1, keepdim=True)
    N = c * ((c * c).mean(-1, keepdim=True) + EPS).rsqrt()
    assert ((dw.double() - (DY * N).sum(0)).abs() <= (190 + n + 8) * 2.0 ** -24 * (DY.abs() * (N.abs() + 1)).sum(0)).all()
    assert ((db.double() - dy.double().sum(0)).abs() <= (2 * n + 8) * 2.0 ** -24 * dy.double().abs().sum(0)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [1, 2, 96, 129, 1024, 1155, 3000, 8191])
def test_sums_that_leave_fp32(dtype, dim):
    check(dtype, dim, (3e38, -3e38, 1e37, -1e36), weights=dim % 2 == 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_infinite_rows_are_not_rows_of_one_value(dtype):
    x = torch.full((3, 200), float("inf"), device="cuda", dtype=TYPE[dtype])
    x[1] = 1.0
    y = torch.empty_like(x)
    B.LayerNorm(LayerNormConfig(200, dtype, EPS)).forward(x, None, None, y)
    assert y[0].isnan().all() and (y[1] == 0).all() and y[2].isnan().all()
