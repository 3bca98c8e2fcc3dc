"""Embedding, norm and head one after the other, their gradients in the units of one plan's gradient buffer, the table of the
embedding and the head's weight apart and tied.  Every stage is held to the 64-bit form of what it was given by the stage
before, within that operator's own bounds."""
import pytest
import torch

from tests import head_reference as H
from tests import layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


@pytest.mark.parametrize("tied", [False, True])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_one_step(tied, grad, kind):
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.head import Head
    from paper_2609_20359_b200.norm import Norm
    from paper_2609_20359_b200.session import Session
    V, d, n = 1501, 136, 300
    shapes = [(V, d), (d,), (d,)] + ([] if tied else [(V, d)])            # table, the norm's weight and bias, the head's weight
    numel = [torch.Size(s).numel() for s in shapes]
    s = Session(sum(numel), numel, groups=1, shard_dim=1, grad_dtype=grad, lr=1e-3)
    g = torch.Generator(device=DEV).manual_seed(1)

    def unit(flat, u):
        off = s.layout["unit_offset"][u]
        return flat[off: off + numel[u]].view(shapes[u])

    p, flat = s.param_bf16[0], s.grads[0][0]
    for u in range(len(shapes)):
        x = torch.randn(shapes[u], generator=g, device=DEV) / (8 if len(shapes[u]) == 2 else 4) + (1.0 if u == 1 else 0.0)
        unit(p, u).copy_(x)
        at = s.layout["unit_shard_offset"][u]
        s.master[0][at: at + numel[u]].copy_(x.flatten())
    flat.fill_(float("nan"))
    head_unit = 0 if tied else 3
    tok = torch.randint(0, 200, (n,), generator=g, device=DEV)            # most rows without a token
    tok[::9] = -100                                                       # padding
    label = torch.randint(0, V, (n,), generator=g, device=DEV)
    label[tok < 0] = -100
    emb, norm, head = Embedding(n, V, d, grad_dtype=grad), Norm(n, d, kind, grad_dtype=grad), Head(n, V, d, grad_dtype=grad)

    x = emb.lookup(tok, unit(p, 0), scale=2.0)
    hidden, mean, rstd = norm.forward(x, unit(p, 1), unit(p, 2))
    grad_hidden = torch.empty_like(hidden)
    loss, lse = head.xent_step(hidden, unit(p, head_unit), label, grad_hidden, unit(flat, head_unit))
    head_grad = unit(flat, head_unit).clone()
    grad_x = norm.backward(x, unit(p, 1), mean, rstd, grad_hidden, unit(flat, 1), unit(flat, 2))
    emb.grad(tok, grad_x, unit(flat, 0), scale=2.0, accumulate=tied)

    assert torch.equal(x, R.lookup(tok, unit(p, 0), 2.0, -100, torch.bfloat16))
    R.check_forward(x, unit(p, 1), unit(p, 2), 1e-5, kind == "rms", hidden, mean, rstd)
    live = label >= 0
    ref = H.with_gradients(hidden, unit(p, head_unit), lambda z: (*H.xent_rows(z, label, live, 0.0, 0.0), live))
    H.check_rows(ref, loss, lse)
    H.check_grads(ref, grad_hidden, head_grad)
    R.check_backward(x, unit(p, 1), mean, rstd, grad_hidden, None, grad_x, unit(flat, 1), unit(flat, 2))
    R.check_embed_grad(unit(flat, 0), tok, grad_x, scale=2.0, old=head_grad if tied else None)
    if not tied:
        assert torch.equal(unit(flat, 3), head_grad)
    before = p.clone()
    s.step()
    torch.cuda.synchronize()
    assert bool(torch.isfinite(s.norms()).all()) and bool(torch.isfinite(p.float()).all()) and not torch.equal(before, p)
    for op in (emb, norm, head, s):
        op.close()


def test_gradient_of_the_chain_against_differences():
    """The whole chain's gradient with respect to one entry of each parameter, in fp32 activations where the operators have
    them: the directional derivative from the kernels' gradients against central differences of the 64-bit loss."""
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.norm import Norm
    V, d, n = 50, 40, 64
    g = torch.Generator(device=DEV).manual_seed(2)
    table = torch.randn(V, d, generator=g, device=DEV).bfloat16()
    w = (1 + 0.2 * torch.randn(d, generator=g, device=DEV)).bfloat16()
    b = (0.1 * torch.randn(d, generator=g, device=DEV)).bfloat16()
    out = torch.randn(n, d, generator=g, device=DEV)                      # the loss is sum(out * y)
    tok = torch.randint(0, V, (n,), generator=g, device=DEV)
    emb = Embedding(n, V, d, act_dtype="f32", grad_dtype="f32")
    norm = Norm(n, d, x_dtype="f32", y_dtype="f32", grad_dtype="f32")
    x = emb.lookup(tok, table)
    _, mean, rstd = norm.forward(x, w, b)
    dw, db, dt = torch.empty(d, device=DEV), torch.empty(d, device=DEV), torch.empty(V, d, device=DEV)
    emb.grad(tok, norm.backward(x, w, mean, rstd, out, dw, db), dt)

    def loss(table, w, b):
        y, _, _ = R.forward(table[tok], w, b, 1e-5, False)
        return (y * out.double()).sum()

    at = [t.double() for t in (table, w, b)]
    for i, grad in enumerate((dt, dw, db)):
        for _ in range(5):
            step = torch.randn(at[i].shape, generator=g, device=DEV, dtype=torch.float64)
            step /= step.norm()
            h = 1e-4
            up, dn = (loss(*(t + k * h * step if j == i else t for j, t in enumerate(at))) for k in (1, -1))
            # central differences: h^2 / 6 of a third derivative of order |out|_1; fp32 gradients: 1e-5 of their norm is 100 roundings
            assert abs(float((up - dn) / (2 * h) - (grad.double() * step).sum())) < 1e-5 * float(grad.double().norm()) + h * h * float(out.abs().sum())


def test_forward_passes_on_two_streams_at_once():
    """Lookups and forward passes have no workspace: calls of one object may overlap."""
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.norm import Norm
    V, d, n = 3000, 1024, 4000
    g = torch.Generator(device=DEV).manual_seed(3)
    table = torch.randn(V, d, generator=g, device=DEV).bfloat16()
    toks = [torch.randint(0, V, (n,), generator=g, device=DEV) for _ in range(2)]
    emb, norm = Embedding(n, V, d, grads=False), Norm(n, d, "rms", grads=False)
    want = [norm.add_forward(emb.lookup(t, table), emb.lookup(t.flip(0), table)) for t in toks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(norm.add_forward(emb.lookup(toks[k], table), emb.lookup(toks[k].flip(0), table)))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            assert all(a is b is None or torch.equal(a, b) for a, b in zip(out, want[k]))


@pytest.mark.parametrize("n", [100, 700, 6000])
def test_two_captured_graphs_with_one_workspace(n):
    """Backward passes of one object captured into two graphs, replayed one after the other in any order."""
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.norm import Norm
    V, d = 900, 256
    g = torch.Generator(device=DEV).manual_seed(4)
    emb, norm = Embedding(n, V, d, grad_dtype="f32"), Norm(n, d, grad_dtype="f32")
    data, graphs = [], []
    for _ in range(2):
        tok = torch.randint(0, 50, (n,), generator=g, device=DEV)
        x, dy = (torch.randn(n, d, generator=g, device=DEV).bfloat16() for _ in range(2))
        _, mean, rstd = norm.forward(x)
        data.append((tok, x, mean, rstd, dy, torch.empty(d, device=DEV), torch.empty(d, device=DEV), torch.empty(V, d, device=DEV),
                     torch.empty_like(x)))

    def step(tok, x, mean, rstd, dy, dw, db, dt, dx):
        norm.backward(x, None, mean, rstd, dy, dw, db, grad_x=dx)
        emb.grad(tok, dx, dt)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for one in data:
            step(*one)
    torch.cuda.current_stream().wait_stream(side)
    for one in data:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*one)
        graphs.append(graph)
    for k in (0, 1, 1, 0, 1):
        for t in data[k][5:]:
            t.fill_(float("nan"))
        graphs[k].replay()
        tok, x, mean, rstd, dy, dw, db, dt, dx = data[k]
        R.check_backward(x, None, mean, rstd, dy, None, dx, dw, db)
        R.check_embed_grad(dt, tok, dx)
    del graphs, graph
