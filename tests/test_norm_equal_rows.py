"""Layer norm of rows whose values are all the same: the variance is nothing but the roundings of fp32, of either sign."""
import pytest
import torch

from tests import layers_reference as R
from tests.test_embed_gpu import DEV, TYPES, gen

pytestmark = pytest.mark.gpu
U = R.U


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def norm(*a, **kw):
    from paper_2609_20359_b200.norm import Norm
    return Norm(*a, device=DEV, **kw)


# few rows, and so many that a thread has several cells; widths that are no power of two, so that 1 / d is rounded
SIZES = [(41, 448), (41, 960), (41, 1000), (41, 1001), (41, 1920), (41, 3584), (41, 3808), (700, 3584), (400, 7168), (5000, 1920), (41, 32768),
         (41, 40000), (3, 65535)]


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("eps", [1e-12, 1e-6, 1e-5])
@pytest.mark.parametrize("n,d", SIZES)
def test_rows_of_equal_values(n, d, eps, x_type):
    g = gen(n + d)
    values = 10.0 ** (3 + 6 * torch.rand(n, generator=g, device=DEV, dtype=torch.float64))
    values[0] = 13033.5439
    values[1::3] *= -1
    x = values.to(TYPES[x_type])[:, None].expand(n, d).contiguous()
    w = 1 + 0.3 * torch.randn(d, generator=g, device=DEV)
    b = 0.2 * torch.randn(d, generator=g, device=DEV)
    op = norm(n, d, "layer", eps, x_type, "f32", "f32", "f32")
    y, mean, rstd = op.forward(x, w, b)
    # A sum's longest chain is K = d / 32 + 16.  The fp32 mean m that is taken off is (K + 2) U |x| from x at most (1 / d and the product
    # are rounded too); every x - m is the same c, without a rounding.  mean(c) and mean(c^2) are off by (K + 2) U and (K + 3) U of
    # themselves, so the variance is off by (3 K + 9) U c^2, and never below zero.  eps, its addition, root and reciprocal: U each.
    K = d / 32 + 16
    m64 = x[:, 0].double()
    c = (K + 2) * U * m64.abs()
    top = eps ** -0.5
    assert bool((rstd.double() <= top * (1 + 4.5 * U)).all()), "the variance is not below zero"
    assert bool((rstd.double() >= (eps + (3 * K + 9) * U * c * c) ** -0.5 * (1 - 4.5 * U)).all())
    R.check("mean", mean, m64, U * m64.abs() + (K + 3) * U * c)
    # the definition gives the bias; c - mean(c) is (K + 2) U c, and two products and two sums round once each
    lim = (w.double().abs() * (top * (K + 5) * U * c)[:, None]) + U * b.double().abs()
    R.check("y", y, b.double().expand(n, d), lim)
    # what the backward pass makes of them is finite in every row's share of the weight's gradient
    dy = torch.randn(n, d, generator=g, device=DEV)
    dw, db = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    dx = op.backward(x, w, mean, rstd, dy, dw, db)
    R.check_backward(x, w, mean, rstd, dy, None, dx, dw, db)


@pytest.mark.parametrize("d", [1000, 40000])
def test_equal_rows_that_are_not_finite(d):
    """NaN and infinite rows stay what they are: no maximum takes them for a variance of zero."""
    op = norm(6, d, "layer", 1e-5, "f32", "f32")
    x = torch.full((6, d), 7.0, device=DEV)
    x[1], x[3], x[4, 5] = float("nan"), float("inf"), float("nan")
    y, mean, rstd = op.forward(x)
    bad = torch.tensor([False, True, False, True, True, False], device=DEV)
    assert torch.equal(y.isnan().all(1), bad) and torch.equal(rstd.isnan(), bad) and bool((y[~bad] == 0).all())
