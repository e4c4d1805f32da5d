"""Layer norm of rows whose mean is far from zero: what the rounding of the mean leaves in the centred values is taken away.

Bounds that belong to the deviations alone, however large the mean.  u = 2^-24, s the row's standard deviation.  Sums run over at most 32 additions one
after the other (16 pairs of a thread, 5 exchanges, 6 of the warps; 32 where values come one by one), so a mean of d values, with its
own two roundings, is 36 u times their mean size off: less than 612 u s where the mean is below 16 deviations, so that no value lies further than 17 s
from zero in the mean.  Rows further out are centred twice more, which leaves 40 u s.  So with a = min(36 mean|x|, 612 s) + 40 s, or 40 s beyond
17 deviations: c is off by u a and a rounding, u |c|; the sum of c^2 by 34 u relatively, the reciprocal root by 21 u with its own error of 4 u, and
n = c r by u (30 |n| + a r).  Backward, with b = 100 + a r and M = mean(|g| (|n| + 1)): mean(g n) is off by b u M, n times it by (b + 30 + a r) u (|n| + 1) M,
mean(g) by 36 u mean |g|, and dx by (2 b + 60) u r (|g| + mean |g| + (|n| + 1) M).  Each result is rounded once more."""
import pytest
import torch

from paper_2604_22808_b200 import binding as B
from paper_2604_22808_b200.configs import LayerNormConfig
from test_layer_norm_equal_rows_gpu import EPS, HALF, TYPE, normal
from test_layer_norm_equal_rows_gpu import check as check_equal_rows

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check(dtype, dim, mean, deviation, eps=EPS, rows=24):
    t, half = TYPE[dtype], HALF[dtype]
    x = (mean + deviation * normal(rows, dim, seed=dim).double()).to(t)
    dy, w, b = normal(rows, dim, seed=dim + 1).to(t), normal(dim, seed=dim + 2), normal(dim, seed=dim + 3)
    norm = B.LayerNorm(LayerNormConfig(dim, dtype, eps))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    norm.forward(x, w, b, y)
    norm.backward(x, w, dy, dx, dw, db)
    X, DY, W = x.double(), dy.double(), w.double()
    c = X - X.mean(-1, keepdim=True)
    var = (c * c).mean(-1, keepdim=True)
    r = (var + norm_eps(eps)).rsqrt()
    n, g = c * r, DY * W
    dev, far = var.sqrt(), X.mean(-1, keepdim=True).abs()
    a = 40 * dev + torch.where(far > 17 * dev, 0, torch.minimum(36 * X.abs().mean(-1, keepdim=True), 612 * dev))
    en = U * (30 * n.abs() + a * r)
    want = n * W + b.double()
    assert ((y.double() - want).abs() <= half * want.abs() + en * W.abs() + 2 * U * ((n * W).abs() + want.abs())).all()
    M = (g.abs() * (n.abs() + 1)).mean(-1, keepdim=True)
    want = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True))
    assert ((dx.double() - want).abs() <= half * want.abs() + (260 + 2 * a * r) * U * r * (g.abs() + g.abs().mean(-1, keepdim=True) + (n.abs() + 1) * M)).all()
    assert ((dw.double() - (DY * n).sum(0)).abs() <= (rows + 8) * U * (DY * n).abs().sum(0) + (DY.abs() * en).sum(0)).all()


def norm_eps(eps):
    return float(torch.tensor(eps, dtype=torch.float32))


@pytest.mark.parametrize("dim", [2, 33, 250, 1001, 1155, 1536, 3001, 5120, 8192])
@pytest.mark.parametrize("mean,deviation", [(1000.0, 0.01), (-1e5, 1.0), (3e7, 2.0), (7.0, 1e-6), (10.0, 1.0), (0.0, 1.0)])
def test_means_of_many_deviations(dim, mean, deviation):
    """fp32, down to rows whose values differ by a few of their last bits."""
    check("fp32", dim, mean, deviation, eps=1e-12)


@pytest.mark.parametrize("dim", [96, 1155, 2050, 4096])
def test_means_of_many_deviations_bf16(dim):
    check("bf16", dim, 300.0, 2.0)
    check("bf16", dim, -3e30, 1e29)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dim", [1, 3, 250, 1155, 1536, 3001, 5120, 8191])
def test_rows_of_one_value(dtype, dim):
    """Whatever the value, y is the bias."""
    check_equal_rows(dtype, dim, (12345.678, -0.1, 1e-10, 1e10, 7e15, -2.5e24, 1e34, 0.0), weights=dim % 2 == 0)
