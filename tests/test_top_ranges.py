"""fls_top_logits where logits over temperature leave the range of fp32 on their way to a log sum exp that does not."""
import pytest
import torch

from tests.test_top_logits import DEV, draw, fls, reference, same  # noqa: F401  (fls builds the library)

pytestmark = pytest.mark.gpu


def check(x, k, T):
    from paper_2609_20359_b200.head import TopLogits
    value, index, lse = TopLogits(x.shape[0], x.shape[1], k)(x, T)
    wv, wi, wl = reference(x, k, T)
    assert torch.equal(index, wi)
    same(value, wv)
    # a difference of logits over T is rounded to 2^-23 of the larger of the two; sums of a few thousand terms; fp32 result
    kept = x.double().masked_fill(x < -1e30, 0.0)
    size = float(kept.abs().max()) / T
    lim = (size * 1.45 + 4) * 2.0 ** -22 + (x.shape[1] / 256 + 20) * 2.0 ** -24 + 2.0 ** -23 * wl.abs()
    assert bool(((lse.double() - wl).abs() <= lim).all())


# parts of a row on several CTAs, rows of 512 and of 256 threads
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V", [(2, 70001), (5, 20000), (320, 30001)])
@pytest.mark.parametrize("low,T", [(-9e36, 0.03), (-9e35, 0.003), (-1e33, 4e-6)])
def test_masks_far_below_at_low_temperature(dtype, n, V, low, T):
    """Whole stretches and whole rows at a large negative value whose product with 1 / T has no fp32."""
    x = T * draw(n, V, torch.float32)
    x[0, : V - 900] = low
    x[1] = low
    x[2:, ::2] = low
    check(x.to(dtype), 8, T)


# from where a rounding of m log2(e) / T was a factor of 2^64 over where it was all of fp32
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V", [(2, 70001), (5, 20000), (320, 30001)])
@pytest.mark.parametrize("level", [3e5, -3e5, 1e9, -1e9, 1e10, -1e10, 1e20, -1e20, 1e30, -1e30])
def test_rows_far_from_zero(dtype, n, V, level):
    """Logits of one magnitude far from zero: all equal, of two values, and a few of another sign."""
    x = torch.full((n, V), level, device=DEV)
    x[0, 17] = 1.5 * level
    x[1, V // 2:] = -level
    from paper_2609_20359_b200.head import TopLogits
    value, index, lse = TopLogits(n, V, 8)(x.to(dtype))
    wv, wi, wl = reference(x.to(dtype), 8, 1.0)
    assert torch.equal(index, wi)
    same(value, wv)
    assert bool(((lse.double() - wl).abs() <= 2.0 ** -22 * wl.abs()).all())


@pytest.mark.parametrize("n,V", [(2, 70001), (320, 30001)])
@pytest.mark.parametrize("T", [1e-38, 1e-39])
def test_lowest_temperatures(n, V, T):
    x = draw(n, V, torch.float32)
    x = x * (2.9e38 * T) / x.abs().max()
    check(x, 8, T)
