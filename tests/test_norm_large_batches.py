"""Norms of batches that give a thread several cells, a warp part of a row and a group of threads many rows, and weights that do
not start on the boundary that the rows start on."""
import pytest
import torch

from tests import layers_reference as R
from tests.test_embed_gpu import DEV, TYPES, gen, outside, rows
from tests.test_norm_gpu import KINDS, PAIRS, norm, params

pytestmark = pytest.mark.gpu

SIZES = [(32773, 768), (16387, 2048), (5003, 512), (4099, 640), (8195, 4096), (2501, 8192), (90001, 64), (40001, 136), (16385, 1001), (301, 12288), (257, 16384)]


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def run(n, d, kind, x_type, y_type, w_type, g_type, residual, pad, shift, off, g):
    """Forward, backward, and what they leave beside their outputs."""
    rms = kind == "rms"
    x, _ = rows(n, d, TYPES[x_type], g, pad, shift, 2.0)
    w, b = params(d, TYPES[w_type], g, True, True)
    if off:
        w, b = (torch.cat([t.new_full((off,), float("nan")), t])[off:] for t in (w, b))
    op = norm(n, d, kind, 1e-5, x_type, y_type, w_type, g_type)
    op.workspace.memory[256:].fill_(255)
    y, flat = rows(n, d, TYPES[y_type], g, pad, shift)
    y.fill_(3.0)
    if residual:
        r, _ = rows(n, d, TYPES[x_type], g, pad, shift)
        want = (x.double() + r.double()).to(TYPES[x_type])
        _, total, mean, rstd = op.add_forward(x, r, w, b, y=y)
        assert torch.equal(total, want)
        x = total
    else:
        _, mean, rstd = op.forward(x, w, b, y=y)
    assert bool(outside(flat, y).isnan().all())
    R.check_forward(x, w, b, 1e-5, rms, y, mean, rstd)
    dy, _ = rows(n, d, TYPES[y_type], g, pad, shift, 1e-2)
    dt = rows(n, d, TYPES[x_type], g, pad, shift, 1e-2)[0] if residual else None
    dx, flat = rows(n, d, TYPES[x_type], g, pad, shift)
    dw, db = (torch.full((d + off,), float("nan"), dtype=TYPES[g_type], device=DEV)[off:] for _ in range(2))
    op.backward(x, w, mean, rstd, dy, dw, db, grad_total=dt, grad_x=dx)
    R.check_backward(x, w, mean, rstd, dy, dt, dx, dw, db)
    assert bool(outside(flat, dx).isnan().all())
    first = dx.clone(), dw.clone(), db.clone()
    op.backward(x, w, mean, rstd, dy, dw, db, grad_total=dt, grad_x=dx)
    assert all(torch.equal(p, q) for p, q in zip(first, (dx, dw, db)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("x_type,y_type", PAIRS)
@pytest.mark.parametrize("n,d", SIZES)
def test_large_batches(n, d, x_type, y_type, kind):
    residual = (n + len(kind)) % 2 == 0 or x_type == y_type == "bf16"
    w_type, g_type = ("f32", "bf16") if (n + d) % 3 == 0 else ("bf16", "f32")
    run(n, d, kind, x_type, y_type, w_type, g_type, residual, 0, 0, 0, gen(n + d))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("x_type,w_type", PAIRS)
@pytest.mark.parametrize("off", [1, 4])
@pytest.mark.parametrize("n,d", [(7, 768), (3001, 768), (40, 4096), (3, 8200), (2, 40000)])
def test_weights_off_a_boundary(n, d, off, x_type, w_type, kind):
    run(n, d, kind, x_type, "bf16", w_type, w_type, n > 10, 0, 0, off, gen(n + d))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,d", [(300, 768), (40, 4096)])
def test_fp32_rows_on_16_byte_boundaries(n, d, kind):
    run(n, d, kind, "f32", "f32", "f32", "f32", True, 4, 4, 0, gen(n + d))
