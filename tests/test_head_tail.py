"""Distillation with the tail as a class where student and teacher disagree about it: a student whose list stands far above
everything else still has a finite loss, and gradients that stay with the columns they belong to."""
import math

import pytest
import torch

from tests import head_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
IGN = -100


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_2609_20359_b200 import build
    build.build()


def far_student(n, V, d, k, gap, T, kind):
    """Logits of the listed columns about `gap` * T above all others; coordinate 0 carries the gap, the others the rest."""
    g = torch.Generator(device=DEV).manual_seed(int(gap) + k)
    h = torch.randn(n, d, generator=g, device=DEV)
    w = torch.randn(V, d, generator=g, device=DEV) * (0.3 * T / math.sqrt(d))
    cols = torch.randperm(V, generator=g, device=DEV)
    h[:, 0], w[:, 0] = 1.0, 0.0
    w[cols[:k], 0] = gap * T - torch.arange(k, device=DEV) * (0.25 * T)
    h, w = h.bfloat16(), w.bfloat16()
    idx = cols[:k].to(torch.int32).expand(n, k).contiguous()
    t = (1.5 * T) * torch.randn(n, k, generator=g, device=DEV)
    tlse = torch.logsumexp(t / T, 1) + 0.1 + torch.rand(n, generator=g, device=DEV)       # the teacher keeps 10 to 66 % outside
    y = torch.randint(0, V, (n,), generator=g, device=DEV)
    if kind != "labels anywhere":
        y = (cols[0] if kind == "labels in the list" else cols[k + 1]).expand(n).contiguous()
    y[1] = IGN
    return h, w, idx, t, tlse, y


def bounds(ref, T):
    """The kernels' e_p at temperature T: the exponent is z / T, its error that of the logit over T."""
    top = float(ref["z_max"]) / T
    ref["e_p"] = 2 * ref["e_z"] / T + (top * 1.45 + 4) * 2.0 ** -22 + 2.0 ** -20
    return ref


def run(n, V, d, k, gap, T, wl, kind, f32=False, piece=0):
    from paper_2609_20359_b200.head import Head
    h, w, idx, t, tlse, y = far_student(n, V, d, k, gap, T, kind)
    gh = torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV)
    gw = torch.full((V, d), math.nan, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    head = Head(n, V, d, top=k, grad_dtype="f32" if f32 else "bf16", piece_bytes=piece)
    loss, lse = head.distill_step(h, w, idx, t, gh, gw, labels=y, teacher_lse=tlse, temperature=T, label_weight=wl)
    ref = R.with_gradients(h, w, lambda z: R.distill_rows(z, idx, t, y, T, 1.0, wl, tlse, IGN))
    ref["z_max"] = (h.double() @ w.double().t()).abs().max()
    bounds(ref, T)
    # q' = 1 - sum q and log q inherit 2^-24 of the teacher's inputs and of its log sum exp, each held in fp32
    R.check_rows(ref, loss, lse, 4 * T * T + wl, T)
    R.check_grads(ref, gh, gw)
    assert head.status() == 0


# from where fp32 lost the tail's gradient (87) over where its coefficient overflowed (89) and the loss was infinite (104) to
# where double has nothing left beside the row's maximum (745)
@pytest.mark.parametrize("T,wl", [(1.0, 0.0), (1.0, 0.5), (0.1, 0.0), (0.25, 0.5)])
@pytest.mark.parametrize("gap", [60, 88, 100, 115, 300, 900])
def test_student_far_above_its_tail(gap, T, wl):
    run(40, 700, 64, 8, gap, T, wl, "labels anywhere")


@pytest.mark.parametrize("kind", ["labels in the list", "labels outside the list"])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("d,piece", [(912, 0), (912, 1 << 20), (64, 1)])
def test_labels_and_both_ways_to_the_logits(kind, f32, d, piece):
    """Kept and formed logits, one and two terms of dL/dz, one and two temperatures."""
    run(150, 1500, d, 20, 120, 1.0, 0.5, kind, f32, piece)
    run(150, 1500, d, 20, 120, 0.25, 0.5, kind, f32, piece)


def test_tail_of_probability_zero():
    """Every column outside the list masked to -inf by the weight: q' > 0 there is an infinite loss by the definition, and
    nothing of it reaches those columns' own gradient."""
    from paper_2609_20359_b200.head import Head
    n, V, d, k = 5, 300, 64, 4
    g = torch.Generator(device=DEV).manual_seed(2)
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, d, generator=g, device=DEV) / 8).bfloat16()
    h[:, 0] = 1.0
    w[k:, 0] = -math.inf
    idx = torch.arange(k, dtype=torch.int32, device=DEV).expand(n, k).contiguous()
    t = torch.randn(n, k, generator=g, device=DEV)
    gw = torch.full((V, d), math.nan, dtype=torch.bfloat16, device=DEV)
    loss, lse = Head(n, V, d, top=k).distill_step(h, w, idx, t, grad_weight=gw, teacher_lse=torch.logsumexp(t, 1) + 0.5)
    assert bool((loss == math.inf).all()) and bool(torch.isfinite(lse).all())
    assert bool((gw[k:] == 0).all()) and bool(torch.isfinite(gw[:k]).all())
