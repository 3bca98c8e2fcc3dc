"""What the two gradients of a head's step owe each other, and where they end."""
import math

import pytest
import torch

from tests import head_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_2609_20359_b200 import build
    build.build()


def make(n, V, d, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV)
    return h, w, y


# formed in several pieces, kept in part, kept altogether, one piece; calls of all rows and of fewer than the head was made for
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,n,V,d,piece", [(400, 400, 6000, 256, 1 << 20), (700, 700, 2500, 320, 1 << 20), (300, 300, 3000, 904, 1 << 22),
                                              (130, 130, 20000, 1024, 0), (64, 64, 40000, 64, 1 << 22), (2000, 700, 9000, 512, 1 << 24)])
def test_one_gradient_alone_has_the_bits_of_both(rows, n, V, d, piece, f32):
    from paper_2609_20359_b200.head import Head
    h, w, y = make(n, V, d)
    head = Head(rows, V, d, grad_dtype="f32" if f32 else "bf16", piece_bytes=piece)

    def buffers():
        return (torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV),
                torch.full((V, d), math.nan, dtype=head.grad_torch_dtype, device=DEV))

    both, alone = buffers(), buffers()
    head.xent_step(h, w, y, *both)
    head.xent_step(h, w, y, grad_hidden=alone[0])
    head.xent_step(h, w, y, grad_weight=alone[1])
    assert torch.equal(alone[0], both[0]) and torch.equal(alone[1], both[1])


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("d,stride", [(1, 8), (23, 24), (34, 40), (67, 72), (100, 104), (125, 128), (126, 136), (71, 96), (64, 72), (1021, 1024)])
def test_nothing_between_the_rows_is_written(d, stride, accumulate, f32):
    """Gradients in views whose rows start on 16-byte boundaries and end anywhere."""
    from paper_2609_20359_b200.head import Head
    n, V = 40, 300
    h, w, y = make(n, V, d)
    dtype = torch.float32 if f32 else torch.bfloat16
    bh = torch.full((n + 1, stride), 5.0, dtype=torch.bfloat16, device=DEV)
    bw = torch.full((V + 1, stride), 5.0, dtype=dtype, device=DEV)
    gh, gw = bh[:n, :d], bw[:V, :d]
    want_h, want_w = torch.empty(n, d, dtype=torch.bfloat16, device=DEV), torch.full((V, d), 5.0, dtype=dtype, device=DEV)
    head = Head(n, V, d, grad_dtype="f32" if f32 else "bf16", any_weight=True)
    head.xent_step(h, w, y, gh, gw, accumulate=accumulate)
    head.xent_step(h, w, y, want_h, want_w, accumulate=accumulate)
    assert torch.equal(gh, want_h) and torch.equal(gw, want_w)
    gh.fill_(5.0)
    gw.fill_(5.0)
    assert bool((bh == 5.0).all()) and bool((bw == 5.0).all())


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n,V,d", [(1, 700, 64), (2, 3000, 256), (1, 12, 1000)])
def test_probabilities_that_cancel(n, V, d, f32):
    """With smoothing p - eps / V may nearly vanish; its error is that of p then, not of the difference."""
    from paper_2609_20359_b200.head import Head
    eps = 0.5
    h, w, y = make(n, V, d)
    gh = torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV)
    gw = torch.full((V, d), math.nan, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    Head(n, V, d, grad_dtype="f32" if f32 else "bf16").xent_step(h, w, y, gh, gw, label_smoothing=eps)
    live = torch.ones(n, dtype=torch.bool, device=DEV)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, eps, 0.0), live))
    p = ref["dz"].abs() + eps / (V * n)                # what the difference is taken of, with the mean's 1 / n
    R.check_grads(ref, gh, None, small=ref["e_p"] * p @ w.double().abs())
    R.check_grads(ref, None, gw, small=ref["e_p"] * p.t() @ h.double().abs())
