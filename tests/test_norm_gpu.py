"""Layer norm and root mean square norm, forward and backward, against plain 64-bit forms."""
import pytest
import torch

from tests import layers_reference as R
from tests.test_embed_gpu import DEV, TYPES, gen, outside, rows

pytestmark = pytest.mark.gpu
KINDS = ["layer", "rms"]
PAIRS = [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")]


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def norm(*a, **kw):
    from paper_2609_20359_b200.norm import Norm
    return Norm(*a, device=DEV, **kw)


SIZES = [
    # n, d, pad, shift
    (1, 1, 0, 0), (1, 2048, 0, 0), (3, 7, 0, 0), (5, 8, 0, 0), (2, 31, 0, 0), (37, 64, 0, 0), (300, 100, 4, 0), (129, 256, 0, 8),
    (1000, 768, 0, 0), (333, 767, 0, 0), (257, 1000, 8, 8), (65, 1001, 0, 1), (2000, 136, 0, 0), (70, 2048, 0, 0), (31, 3001, 0, 3),
    (40, 4096, 0, 0), (9, 5000, 0, 0), (17, 8192, 0, 0), (3, 12345, 0, 0), (5, 16384, 0, 0), (2, 16392, 0, 0), (3, 32768, 0, 0),
    (2, 32769, 0, 0), (2, 65536, 0, 0), (20000, 64, 0, 0), (5000, 8, 0, 0), (10000, 3, 0, 0)]


def params(d, dtype, g, weight, bias):
    w = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dtype) if weight else None
    b = (0.2 * torch.randn(d, generator=g, device=DEV)).to(dtype) if bias else None
    return w, b


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_forward(kind, x_type, y_type, n, d, pad, shift):
    g = gen(n + d)
    wt = "f32" if (n + d) % 3 == 0 else "bf16"
    x, _ = rows(n, d, TYPES[x_type], g, pad, shift, 2.0)
    w, b = params(d, TYPES[wt], g, True, kind == "layer")
    y, flat = rows(n, d, TYPES[y_type], g, pad, shift)
    y.fill_(3.0)
    op = norm(n, d, kind, 1e-5, x_type, y_type, wt, grads=False)
    got, mean, rstd = op.forward(x, w, b, y=y)
    assert got is y and (mean is None) == (kind == "rms") and bool(outside(flat, y).isnan().all())
    R.check_forward(x, w, b, 1e-5, kind == "rms", y, mean, rstd)
    again, none, no = op.forward(x, w, b, stats=False)
    assert none is None and no is None and torch.equal(again, y)
    # without weight and bias
    got, mean, rstd = op.forward(x)
    R.check_forward(x, None, None, 1e-5, kind == "rms", got, mean, rstd)
    # with a residual
    r, _ = rows(n, d, TYPES[x_type], g, pad, shift)
    want = (x.double() + r.double()).to(TYPES[x_type])
    total, flat = rows(n, d, TYPES[x_type], g, pad, shift)
    got, out, mean, rstd = op.add_forward(x, r, w, b, total=total)
    assert out is total and torch.equal(total, want) and bool(outside(flat, total).isnan().all())
    R.check_forward(want, w, b, 1e-5, kind == "rms", got, mean, rstd)
    # in place of either
    for into in (r, x):
        a, c = (x, r) if into is r else (x, (want.double() - x.double()).to(TYPES[x_type]))
        expect = (a.double() + c.double()).to(TYPES[x_type])
        got, out, _, _ = op.add_forward(a, c, w, b, total=into)
        assert out is into and torch.equal(into, expect)
        R.check_forward(expect, w, b, 1e-5, kind == "rms", got, None, None)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("n,d,pad,shift", SIZES)
def test_backward(kind, x_type, y_type, n, d, pad, shift):
    g = gen(n + d)
    rms = kind == "rms"
    wt, gt = ("f32", "bf16") if (n + d) % 3 == 0 else ("bf16", "f32")
    x, _ = rows(n, d, TYPES[x_type], g, pad, shift, 2.0)
    w, _ = params(d, TYPES[wt], g, True, False)
    dy, _ = rows(n, d, TYPES[y_type], g, pad, shift, 1e-2)
    dt, _ = rows(n, d, TYPES[x_type], g, pad, shift, 1e-2)
    mean, rstd = (t.float() for t in R.statistics(x.double(), 1e-5, rms))
    mean = None if rms else mean
    op = norm(n, d, kind, 1e-5, x_type, y_type, wt, gt)
    op.workspace.memory[256:].fill_(255)
    dw, db = (torch.full((d,), float("nan"), dtype=TYPES[gt], device=DEV) for _ in range(2))
    dx, flat = rows(n, d, TYPES[x_type], g, pad, shift)
    got = op.backward(x, w, mean, rstd, dy, dw, db, grad_x=dx)
    assert got is dx and bool(outside(flat, dx).isnan().all())
    R.check_backward(x, w, mean, rstd, dy, None, dx, dw, db)
    # the same bits every time, and whichever gradients are asked for
    first = dx.clone(), dw.clone(), db.clone()
    dx2 = op.backward(x, w, mean, rstd, dy)
    assert torch.equal(dx2, first[0])
    dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
    assert op.backward(x, w, mean, rstd, dy, dw2, input_grad=False) is None
    R.check_backward(x, w, mean, rstd, dy, grad_weight=dw2)
    op.backward(x, w, mean, rstd, dy, None, db2)
    R.check_backward(x, w, mean, rstd, dy, grad_bias=db2)
    op.backward(x, w, mean, rstd, dy, dw, db, grad_x=dx)
    assert torch.equal(dx, first[0]) and torch.equal(dw, first[1]) and torch.equal(db, first[2])
    # the residual's gradient, in place too; sums on top of what is there
    old = [torch.randn(d, generator=g, device=DEV).to(TYPES[gt]) for _ in range(2)]
    dw.copy_(old[0]); db.copy_(old[1])
    got = op.backward(x, w, mean, rstd, dy, dw, db, grad_total=dt, accumulate=True)
    R.check_backward(x, w, mean, rstd, dy, dt, got, dw, db, *old)
    before = dt.clone()
    assert op.backward(x, None, mean, rstd, dy, grad_total=dt, grad_x=dt) is dt
    R.check_backward(x, None, mean, rstd, dy, before, dt)


@pytest.mark.parametrize("kind", KINDS)
def test_no_rows(kind):
    op = norm(4, 16, kind, grad_dtype="f32")
    x = torch.empty(0, 16, dtype=torch.bfloat16, device=DEV)
    y, total, mean, rstd = op.add_forward(x, x)
    assert y.shape == total.shape == (0, 16) and rstd.shape == (0,)
    dw, db = torch.ones(16, device=DEV), torch.ones(16, device=DEV)
    assert op.backward(x, None, mean, rstd, x, dw, db, accumulate=True).shape == (0, 16)
    assert bool((dw == 1).all()) and bool((db == 1).all())
    op.backward(x, None, mean, rstd, x, dw, db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 100, 768, 2048, 8200])
@pytest.mark.parametrize("centre,spread", [(1e4, 1.0), (-300.0, 1e-2), (0.0, 1e-6), (0.0, 1e6), (5.0, 0.0)])
def test_rows_far_from_zero_and_of_any_size(kind, d, centre, spread):
    """fp32 rows whose mean is far larger than what varies; rows of equal values; rows as small as eps."""
    g = gen(d)
    n = 33
    x = centre + spread * torch.randn(n, d, generator=g, device=DEV)
    w, b = params(d, torch.float32, g, True, True)
    op = norm(n, d, kind, 1e-5, "f32", "f32", "f32", "f32")
    y, mean, rstd = op.forward(x, w, b)
    R.check_forward(x, w, b, 1e-5, kind == "rms", y, mean, rstd)
    dy = torch.randn(n, d, generator=g, device=DEV)
    dw, db = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    dx = op.backward(x, w, mean, rstd, dy, dw, db)
    R.check_backward(x, w, mean, rstd, dy, None, dx, dw, db)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [96, 1000, 1003, 40000])
def test_a_row_that_is_not_finite_stays_alone(kind, d):
    n = 40
    g = gen(d)
    op = norm(n, d, kind)
    x = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    good, _, _ = op.forward(x)
    bad = x.clone()
    bad[7, d // 2], bad[20, 0], bad[39, d - 1] = float("nan"), float("inf"), float("-inf")
    y, mean, rstd = op.forward(bad)
    hit = torch.zeros(n, dtype=torch.bool, device=DEV)
    hit[[7, 20, 39]] = True
    assert torch.equal(y[~hit], good[~hit]) and bool(y[hit].isnan().any(1).all()) and bool(rstd[~hit].isfinite().all())
    dy = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    dx = op.backward(bad, None, mean, rstd, dy)
    want = op.backward(x, None, *(t for t in op.forward(x)[1:]), dy)
    assert torch.equal(dx[~hit], want[~hit])


def test_eps_zero_and_large():
    x = torch.randn(10, 64, generator=gen(0), device=DEV)
    for eps in (0.0, 1.0, 1e6):
        for kind in KINDS:
            op = norm(10, 64, kind, eps, "f32", "f32")
            y, mean, rstd = op.forward(x)
            R.check_forward(x, None, None, eps, kind == "rms", y, mean, rstd)


def test_many_rows_beyond_32_bits():
    """Rows that start beyond 2^32 elements."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    d, n = 64, 3
    flat = torch.zeros((1 << 32) + 1024, dtype=torch.bfloat16, device=DEV)
    stride = (1 << 31) - 8
    x = flat.as_strided((n, d), (stride, 1))
    x.copy_(torch.randn(n, d, generator=gen(1), device=DEV))
    other = torch.zeros_like(flat)
    y = other.as_strided((n, d), (stride, 1))
    op = norm(n, d, "layer", grad_dtype="f32")
    _, mean, rstd = op.forward(x, y=y)
    R.check_forward(x, None, None, 1e-5, False, y, mean, rstd)
    dy = torch.randn(n, d, generator=gen(2), device=DEV).bfloat16()
    dw = torch.empty(d, device=DEV)
    op.backward(x, None, mean, rstd, dy, dw, grad_x=y)
    R.check_backward(x, None, mean, rstd, dy, None, y, dw)


@pytest.mark.parametrize("kind", KINDS)
def test_captured_and_replayed(kind):
    n, d = 500, 768
    g = gen(3)
    op = norm(n, d, kind, grad_dtype="f32")
    x, r, dy = (rows(n, d, torch.bfloat16, g)[0] for _ in range(3))
    w, b = params(d, torch.bfloat16, g, True, True)
    dw, db = torch.empty(d, device=DEV), torch.empty(d, device=DEV)

    def step():
        y, total, mean, rstd = op.add_forward(x, r, w, b)
        dx = op.backward(total, w, mean, rstd, dy, dw, db)
        return y, total, mean, rstd, dx

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, total, mean, rstd, dx = step()
    for seed in (4, 5):
        h = gen(seed)
        x.copy_(torch.randn(n, d, generator=h, device=DEV))
        dy.copy_(torch.randn(n, d, generator=h, device=DEV))
        graph.replay()
        R.check_forward((x.double() + r.double()).bfloat16(), w, b, 1e-5, kind == "rms", y, mean, rstd)
        R.check_backward(total, w, mean, rstd, dy, None, dx, dw, db)
    del graph


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_on_another_stream(how):
    n, d = 3000, 1024
    g = gen(6)
    x, dy = (rows(n, d, torch.bfloat16, g)[0] for _ in range(2))
    op = norm(n, d, "layer", grad_dtype="f32")
    late_x, late_dy = torch.zeros_like(x), torch.zeros_like(dy)
    dw = torch.empty(d, device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        late_x.copy_(x)
        late_dy.copy_(dy)
    kw = dict(stream=s if how == "stream" else s.cuda_stream) if how != "current" else {}
    with torch.cuda.stream(s if how == "current" else torch.cuda.default_stream()):
        y, mean, rstd = op.forward(late_x, **kw)
        dx = op.backward(late_x, None, mean, rstd, late_dy, dw, **kw)
    torch.cuda.synchronize()
    R.check_forward(x, None, None, 1e-5, False, y, mean, rstd)
    R.check_backward(x, None, mean, rstd, dy, None, dx, dw)


def test_refusals():
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.norm import Norm
    op = norm(8, 16)
    x = torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV)
    one = torch.zeros(16, dtype=torch.bfloat16, device=DEV)
    st = torch.zeros(8, device=DEV)
    for bad in (lambda: op.forward(x.float()), lambda: op.forward(x[:, :8]), lambda: op.forward(x.cpu()), lambda: op.forward(x, one.float()),
                lambda: op.forward(x, one[:8]), lambda: op.forward(x, y=x.float()), lambda: op.add_forward(x, x[:7]),
                lambda: op.backward(x, None, None, st, x), lambda: op.backward(x, None, st, None, x), lambda: op.backward(x, None, st, st[:7], x),
                lambda: norm(8, 16, "rms").backward(x, None, st, st, x), lambda: op.backward(x, None, st, st, x, one.float()),
                lambda: op.backward(x, None, st, st, x, grad_total=x, input_grad=False), lambda: op.backward(x, None, st, st, x[:1].expand(8, 16)),
                lambda: Norm(8, 16, "batch"), lambda: Norm(8, 16, x_dtype="f16")):
        with pytest.raises(ValueError):
            bad()

    def refused(code, f, *a, **kw):
        with pytest.raises(fls.FlsError) as err:
            f(*a, **kw)
        assert err.value.code == code

    more = torch.zeros(9, 16, dtype=torch.bfloat16, device=DEV)
    refused(fls.FLS_EINVAL, op.forward, more)
    refused(fls.FLS_EINVAL, norm(8, 16, grads=False).backward, x, None, st, st, x)
    refused(fls.FLS_EPTR, op.forward, x, y=x)
    refused(fls.FLS_EPTR, op.add_forward, x, x.clone(), y=more[:8], total=more[1:])
    refused(fls.FLS_EPTR, op.add_forward, more[:8], x, total=more[1:])                # overlaps, but is not the same
    refused(fls.FLS_EPTR, op.backward, x, None, st, st, x.clone(), grad_x=x)
    refused(fls.FLS_EPTR, op.backward, x, None, st, st, more[:8], grad_x=more[1:])
    refused(fls.FLS_EPTR, op.backward, x, None, st, st, x, one, one)
    torch.cuda.synchronize()
