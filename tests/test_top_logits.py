"""fls_top_logits: refusals on the CPU; values, indices (ties to the lowest) and log sum exp on the GPU."""
import math

import pytest
import torch

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def fls():
    from paper_2609_20359_b200 import build
    build.build()
    import paper_2609_20359_b200._binding as b
    return b


@pytest.mark.parametrize("kw,code", [(dict(logit_dtype=2), "FLS_EINVAL"), (dict(vocab=0), "FLS_EINVAL"), (dict(top=0), "FLS_EINVAL"),
                                     (dict(top=129), "FLS_EINVAL"), (dict(temperature=0.0), "FLS_EINVAL"), (dict(stride=99), "FLS_EINVAL"),
                                     (dict(temperature=math.nan), "FLS_EINVAL"), (dict(rows=1 << 25), "FLS_EINVAL"),
                                     (dict(logits=0), "FLS_EPTR"), (dict(logits=3), "FLS_EALIGN")])
def test_refuses(fls, kw, code):
    base = dict(logits=256, logit_dtype=fls.FLS_GRAD_BF16, rows=2, vocab=100, stride=0, top=5, temperature=1.0, value=256, index=256, lse=256)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_top_logits(**{**base, **kw}, stream=0)
    assert e.value.code == getattr(fls, code)


def test_no_rows_is_nothing_to_do(fls):
    fls.fls_top_logits(0, fls.FLS_GRAD_BF16, 0, 100, 0, 5, 1.0, 0, 0, 0, stream=0)


def reference(x, k, T):
    """Stable descending order of 64-bit values (NaN first, -inf never), one row after the other."""
    z = x.double()
    rank = torch.where(torch.isnan(z), math.inf, z)
    n, V = z.shape
    nan_first = torch.argsort(torch.isnan(z).int(), dim=1, descending=True, stable=True)
    order = nan_first.gather(1, torch.argsort(-rank.gather(1, nan_first), dim=1, stable=True))[:, :k]
    value = z.gather(1, order)
    index = order.to(torch.int32)
    index[value == -math.inf] = -1
    if k > V:
        value = torch.nn.functional.pad(value, (0, k - V), value=-math.inf)
        index = torch.nn.functional.pad(index, (0, k - V), value=-1)
    return value, index, torch.logsumexp(z / T, 1)


def same(a, b):
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)].double(), b[~torch.isnan(b)].double())


def check(x, k, T=1.0):
    from paper_2609_20359_b200.head import TopLogits
    value, index, lse = TopLogits(x.shape[0], x.shape[1], k)(x, T)
    wv, wi, wl = reference(x, k, T)
    assert torch.equal(index, wi)
    same(value, wv)
    fin = torch.isfinite(wl)
    same(lse[~fin], wl[~fin])
    # 2^x of a rounded argument (2^-23 of |x| log2(e) / T), sums of V / 512 terms per thread and a tree, fp32 result
    size = float(x.float().abs().masked_fill(~torch.isfinite(x), 0).max()) / T if x.numel() else 0.0
    lim = (size * 1.45 + 4) * 2.0 ** -22 + (x.shape[1] / 512 + 20) * 2.0 ** -24 + 2.0 ** -23 * wl[fin].abs()
    assert bool(((lse[fin].double() - wl[fin]).abs() <= lim).all())


def draw(n, V, dtype, seed=0, scale=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(n, V, generator=g, device=DEV)).to(dtype)


# rows that share a cluster of 1, 2, 4 and 8 CTAs; rows of one element to many vectors per thread; unaligned odd rows
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 5, 8), (2, 7, 7), (5, 129, 128), (4, 1000, 128), (1, 4096, 1), (2, 8191, 64), (3, 8193, 64),
                                   (1, 50257, 20), (37, 33333, 33), (40, 32768, 64), (80, 20001, 5), (150, 9000, 100), (300, 4099, 64),
                                   (1, 128256, 128), (200, 128256, 64)])
def test_sizes(dtype, n, V, k):
    check(draw(n, V, dtype, n + V), k, 1.0 if n % 2 else 2.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [1, 4, 310])
@pytest.mark.parametrize("kind", ["equal", "two values", "rising", "falling", "zeros of both signs", "steps", "one block"])
def test_ties_and_orders(dtype, n, kind):
    V = 40001
    x = torch.zeros(n, V, device=DEV)
    i = torch.arange(V, device=DEV)
    if kind == "equal":
        x += 3.25
    elif kind == "two values":
        x[:, 1::3] = 1.0
    elif kind == "rising":
        x += i * 2.0 ** -10
    elif kind == "falling":
        x -= i * 2.0 ** -10
    elif kind == "zeros of both signs":
        x[:, ::2] = -0.0
    elif kind == "steps":
        x += (i * 7919 % 50) / 8
    else:
        x[:, 20000:23000] = 5.0 + (i[:3000] % 11)
    check(x.to(dtype), 64)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V", [(1, 300001), (20, 70001), (30, 140003)])
def test_rows_shared_by_a_cluster(dtype, n, V):
    """Long rows of few are cut into 2, 4 or 8 parts: ties, masks and the sum have to hold across the cuts."""
    check(draw(n, V, dtype), 77, 1.5)
    x = torch.zeros(n, V, device=DEV)
    x[:, ::3] = -math.inf
    x[:, V // 2 - 20: V // 2 + 20] = 2.0
    check(x.to(dtype), 64)
    x[:] = -math.inf
    x[:, -3:] = 1.0
    check(x.to(dtype), 8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [2, 320])
def test_masked_and_special_values(dtype, n):
    V, k = 30001, 16
    x = draw(n, V, dtype)
    x[0] = -math.inf                                   # nothing to choose
    x[1, 5:] = -math.inf                               # fewer than k
    check(x, k)
    x[0, 30000] = 1.0
    x[1, 7] = torch.finfo(dtype).min                   # the lowest value is still a value
    x[1, 9] = torch.finfo(dtype).max
    check(x, k)
    x[0, 12345] = math.inf
    x[1, 3] = math.nan
    x[1, 20000] = math.nan
    check(x, k)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [2, 320])
def test_masks_of_the_lowest_value(dtype, n):
    """Whole stretches of a row, and whole rows, at the type's lowest value."""
    V, k = 20000, 8
    low = torch.finfo(dtype).min
    x = draw(n, V, dtype)
    x[0] = low
    x[1, :19000] = low
    from paper_2609_20359_b200.head import TopLogits
    value, index, lse = TopLogits(n, V, k)(x)
    wv, wi, wl = reference(x, k, 1.0)
    assert torch.equal(index, wi) and torch.equal(value.double(), wv)
    assert float(lse[0]) == low                        # log V is far below its last digit
    assert bool(((lse[1:].double() - wl[1:]).abs() <= 2e-6 * wl[1:].abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("off,extra", [(1, 0), (3, 5), (0, 8)])
def test_strides(off, extra):
    n, V = 9, 5001
    for dtype in (torch.bfloat16, torch.float32):
        buf = torch.full((off + n * (V + extra),), 100.0, dtype=dtype, device=DEV)
        x = buf[off:].view(n, V + extra)[:, :V]
        x.copy_(draw(n, V, dtype))
        check(x, 30)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    from paper_2609_20359_b200.head import TopLogits
    n, V, k = 20000, 120001, 8
    x = torch.zeros(n, V, dtype=torch.bfloat16, device=DEV)
    x[-5:] = draw(5, V, torch.bfloat16)
    x[9000] = draw(1, V, torch.bfloat16, 1)[0]
    value, index, _ = TopLogits(n, V, k)(x)
    for rows in (slice(n - 5, n), slice(9000, 9001), slice(0, 2)):
        wv, wi, _ = reference(x[rows], k, 1.0)
        assert torch.equal(index[rows], wi) and torch.equal(value[rows].double(), wv)


@pytest.mark.gpu
def test_feeds_distillation():
    """values, indices and lse of a teacher go into the loss as they are; a student equal to its teacher has KL 0."""
    from paper_2609_20359_b200.head import Head, TopLogits
    g = torch.Generator(device=DEV).manual_seed(1)
    n, V, d, k, T = 50, 3000, 64, 32, 2.0
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, d, generator=g, device=DEV) / 4).bfloat16()
    z = h.float() @ w.float().t()
    value, index, lse = TopLogits(n, V, k)(z, T)
    for tl in (lse, None):
        gh = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
        loss, _ = Head(n, V, d, top=k).distill_step(h, w, index, value, gh, teacher_lse=tl, temperature=T, row_weight=torch.ones(n, device=DEV))
        p = torch.softmax(z.double() / T, 1)
        inside = p.gather(1, index.long())
        # with the tail as a class both sides agree; renormalised, KL = -log of the student's mass on the list
        want = torch.zeros(n, device=DEV, dtype=torch.float64) if tl is not None else -T * T * torch.log(inside.sum(1))
        assert bool(((loss.double() - want).abs() <= 2e-4).all())
        if tl is not None:
            assert float(gh.float().abs().max()) <= 2e-4


@pytest.mark.gpu
def test_stream_and_refusals_on_the_device(fls):
    from paper_2609_20359_b200.head import TopLogits
    top = TopLogits(4, 1000, 10)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        x = draw(4, 1000, torch.float32)
    value, index, _ = top(x, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(index, reference(x, 10, 1.0)[1])
    with pytest.raises(ValueError):
        top(x[:, :999])
    with pytest.raises(ValueError):
        top(x.half())
    with pytest.raises(ValueError):
        top(torch.empty(5, 1000, device=DEV))
    with pytest.raises(ValueError):
        TopLogits(4, 1000, 129)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_top_logits(x, fls.FLS_GRAD_F32, 4, 1000, 0, 10, 1.0, value, x, value)
    assert e.value.code == fls.FLS_EPTR
