"""The head where logits are far from zero: columns masked through the weight, and rows whose logits are all large."""
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


def masked(n, V, d, level, first, seed=0):
    """Coordinate 0 of every hidden state is 1 and of the weight's rows from `first` on `level`: a bias that masks them."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(n, d, generator=g, device=DEV)
    w = torch.randn(V, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))
    h[:, 0], w[:, 0] = 1.0, 0.0
    w[first:, 0] = level
    y = torch.randint(0, first, (n,), generator=g, device=DEV)
    y[0] = -100
    return h.bfloat16(), w.bfloat16(), y, g


LEVELS = [-1e4, -1e6, -1e10, -1e30, float(torch.finfo(torch.bfloat16).min), -math.inf]


# n and d: logits kept, and formed twice; one row tile that ends among the rows, two terms of dL/dz
@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("n,d,f32", [(40, 128, False), (300, 64, False), (300, 64, True), (200, 1024, True)])
def test_columns_masked_through_the_weight(n, d, f32, level):
    """Masked columns have probability zero: losses and gradients are those of the vocabulary without them.  (Their hidden
    gradient is 0 times the mask, which is NaN for -inf in any form; only the weight's is asked for then.)"""
    from paper_2609_20359_b200.head import Head
    V, first = 1200, 700                              # whole 128-column stretches masked, and one in part
    h, w, y, _ = masked(n, V, d, level, first)
    finite = level != -math.inf
    gh = torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV) if finite else None
    gw = torch.full((V, d), math.nan, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    head = Head(n, V, d, grad_dtype="f32" if f32 else "bf16")
    loss, lse = head.xent_step(h, w, y, gh, gw, z_loss=1e-3)
    live = y >= 0
    ref = R.with_gradients(h, w[:first], lambda z: (*R.xent_rows(z, y, live, 0.0, 1e-3), live))
    R.check_rows(ref, loss, lse, 1 + 2e-3 * float(ref["lse"].max()))
    R.check_grads(ref, gh, gw[:first])
    assert bool((gw[first:] == 0).all()) and head.status() == 0


@pytest.mark.parametrize("level", LEVELS)
@pytest.mark.parametrize("T,wl", [(1.0, 0.0), (0.25, 0.0), (2.0, 0.5)])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,d", [(40, 128), (300, 64)])
def test_distillation_with_masked_columns(n, d, tail, T, wl, level):
    from paper_2609_20359_b200.head import Head
    V, first, k = 1200, 700, 12
    h, w, y, g = masked(n, V, d, level, first)
    idx = torch.stack([torch.randperm(first, generator=g, device=DEV)[:k] for _ in range(n)]).to(torch.int32)
    t = torch.randn(n, k, generator=g, device=DEV)
    tlse = torch.logsumexp(t / T, 1) + 0.5 if tail else None
    gw = torch.full((V, d), math.nan, dtype=torch.bfloat16, device=DEV)
    loss, lse = Head(n, V, d, top=k).distill_step(h, w, idx, t, grad_weight=gw, labels=y, teacher_lse=tlse, temperature=T, label_weight=wl)
    ref = R.with_gradients(h, w[:first], lambda z: R.distill_rows(z, idx, t, y, T, 1.0, wl, tlse, -100))
    top = float((h.double() @ w[:first].double().t()).abs().max()) / T
    ref["e_p"] = 2 * ref["e_z"] / T + (top * 1.45 + 4) * 2.0 ** -22 + 2.0 ** -20
    R.check_rows(ref, loss, lse, (12 if tail else 4) * T * T + wl, T)
    # p' - q' of the tail: both are below 1 and p' is known to e_p
    R.check_grads(ref, None, gw[:first], small=ref["e_p"] * T * float(h.float().abs().max()) if tail else 0.0)
    assert bool((gw[first:] == 0).all())


@pytest.mark.parametrize("level", [1e5, -1e5, 1e9, -1e9, 1e12, -1e12, 1e30, -1e30])
@pytest.mark.parametrize("n,d", [(40, 128), (300, 64)])
def test_rows_far_from_zero(n, d, level):
    """Every logit at one large magnitude.  They are equal there to fp32's last digit, so the loss is known to that only; it
    and all gradients are finite, and dL/dz stays within what probabilities allow."""
    from paper_2609_20359_b200.head import Head
    V = 700
    h, w, y, _ = masked(n, V, d, 0.0, V)
    w[:, 0] = level
    gh = torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV)
    gw = torch.full((V, d), math.nan, dtype=torch.bfloat16, device=DEV)
    loss, lse = Head(n, V, d).xent_step(h, w, y, gh, gw, row_weight=torch.ones(n, device=DEV))
    live = y >= 0
    z = h.double() @ w.double().t()
    ulp = 2.0 ** -20 * z.abs().max()
    want = torch.where(live, torch.logsumexp(z, 1), 0.0)
    assert bool(((lse.double() - want).abs() <= ulp).all())
    assert bool(((loss.double() - torch.where(live, want - z.gather(1, y.clamp_min(0)[:, None])[:, 0], 0.0)).abs() <= ulp).all())
    # |dL/dz| <= 1 in every element, bf16 sums
    assert bool((gw.float().abs() <= 1.01 * h.float().abs().sum(0)).all())
    assert bool((gh.float().abs() <= 1.01 * V * w.float().abs().max()).all())
