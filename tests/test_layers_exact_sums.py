"""Gradients whose sums are whole numbers that fp32 holds exactly: any order gives the same bits, and a term that is lost, taken
twice or put into another row shows, however many there are."""
import pytest
import torch

from tests.test_embed_gpu import DEV, TYPES, embedding, gen, outside, rows, tokens_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def whole(shape, largest, dtype, g):
    return torch.randint(-largest, largest + 1, shape, generator=g, device=DEV).to(dtype)


# ------------------------------------------------------------------------------------------------ embedding
# Up to 300000 terms of at most 7, added to what is there: below 2^24 in size, so every partial sum is exact.
EMBED = [(4096, 1031, 256), (4096, 5003, 768), (8191, 3001, 1000), (8193, 700, 33), (16384, 511, 64), (16385, 3, 264), (70000, 3, 24), (70000, 9001, 136),
         (131072, 7, 40), (131073, 5003, 16), (300000, 3, 9), (300000, 70001, 8), (257, 3, 520), (512, 40, 1000), (511, 2, 96), (513, 61, 72), (2048, 2, 300),
         (2049, 97, 776), (700, 90001, 256)]


@pytest.mark.parametrize("act,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("kind", ["same", "few", "text", "mixed"])
@pytest.mark.parametrize("n,V,d", EMBED)
def test_embedding_gradient(n, V, d, kind, act, grad):
    g = gen(n + V + d)
    tok = tokens_of(kind, n, V, g)
    dy = whole((n, d), 7, TYPES[act], g)
    live = (tok >= 0) & (tok < V)
    want = torch.zeros(V, d, dtype=torch.float64, device=DEV).index_add_(0, tok[live], dy[live].double())
    e = embedding(n, V, d, act_dtype=act, grad_dtype=grad)
    gw, flat = rows(V, d, TYPES[grad], g, 8 if n % 2 else 0, 8 if n % 2 else 0)
    gw.fill_(float("nan"))
    e.grad(tok, dy, gw, scale=2.0)                                         # a power of two: exact
    assert torch.equal(gw, (2.0 * want).to(gw.dtype))
    old = whole((V, d), 100, TYPES[grad], g)
    gw.copy_(old)
    e.grad(tok, dy, gw, accumulate=True)
    assert torch.equal(gw, (old.double() + want).to(gw.dtype)) and bool(outside(flat, gw).isnan().all())


# ------------------------------------------------------------------------------------------------ norms
# Whole x, mean and grad_y and a deviation of 1: terms of at most 7 * 8.  rows x 56 stays below 2^24.
NORM = [(32773, 768), (16387, 2048), (5003, 512), (4099, 640), (8195, 4096), (2501, 8192), (90001, 64), (90001, 60), (40001, 333), (16389, 1001), (4100, 2564),
        (1023, 4096), (300, 8200), (3001, 12288), (700, 16385), (97, 65536), (1, 768), (2, 2304), (149, 3000)]


@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("n,d", NORM)
def test_norm_gradients(n, d, kind, x_type, y_type):
    from paper_2609_20359_b200.norm import Norm
    g = gen(n + d)
    grad = "bf16" if (n + d) % 3 == 0 else "f32"
    x, dy = whole((n, d), 7, TYPES[x_type], g), whole((n, d), 7, TYPES[y_type], g)
    mean = whole((n,), 1, torch.float32, g) if kind == "layer" else None
    rstd = torch.ones(n, device=DEV)
    xh = x.float() if mean is None else x.float() - mean[:, None]
    dw, db = torch.zeros(d, dtype=torch.float64, device=DEV), torch.zeros(d, dtype=torch.float64, device=DEV)
    for lo in range(0, n, 8192):
        p = dy[lo: lo + 8192].double()
        dw += (p * xh[lo: lo + 8192].double()).sum(0)
        db += p.sum(0)
    op = Norm(n, d, kind, x_dtype=x_type, y_dtype=y_type, grad_dtype=grad, device=DEV)
    op.workspace.memory[256:].fill_(255)
    old = [whole((d,), 100, TYPES[grad], g) for _ in range(2)]
    for into in (True, False):                                             # with and without the gradient of x
        gw, gb = (torch.full((d,), float("nan"), dtype=TYPES[grad], device=DEV) for _ in range(2))
        op.backward(x, None, mean, rstd, dy, gw, gb, input_grad=into)
        assert torch.equal(gw, dw.to(gw.dtype)) and torch.equal(gb, db.to(gb.dtype))
        gw.copy_(old[0]); gb.copy_(old[1])
        op.backward(x, None, mean, rstd, dy, gw, gb, input_grad=into, accumulate=True)
        assert torch.equal(gw, (old[0].double() + dw).to(gw.dtype)) and torch.equal(gb, (old[1].double() + db).to(gb.dtype))
