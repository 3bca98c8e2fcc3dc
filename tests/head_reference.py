"""Plain 64-bit forms of the head losses (gradients by autograd) and the error bounds the kernels are held to."""
from __future__ import annotations

import math

import torch


def xent_rows(z, y, live, eps, zeta):
    lse = torch.logsumexp(z, 1)
    nll = lse - z.gather(1, y.clamp(0, z.shape[1] - 1)[:, None])[:, 0]
    loss = (1 - eps) * nll + zeta * lse * lse
    if eps:
        loss = loss + eps * (lse - z.mean(1))
    return torch.where(live, loss, 0.0), torch.where(live, lse, 0.0)


def distill_rows(z, idx, top, y, T, wd, wl, tlse, ignore):
    """Row by row from the definition; returns (loss, lse, live)."""
    V = z.shape[1]
    losses, lses, live = [], [], []
    for n in range(z.shape[0]):
        has = (idx[n] >= 0) & (idx[n] < V) & (top[n] != -math.inf)
        cols, t = idx[n][has].long(), top[n][has].double() / T
        labelled = bool(wl) and int(y[n]) != ignore
        zt = z[n] / T
        lse = torch.logsumexp(zt, 0)
        loss = z.new_zeros(())
        if len(cols):
            logq = torch.log_softmax(t, 0) if tlse is None else t - tlse[n].double()
            q = torch.exp(logq)
            part = torch.where(q > 0, q * (logq - (zt[cols] - lse)), 0.0).sum()
            if tlse is not None:
                rest = max(0.0, 1.0 - float(q.sum()))
                if rest > 0:
                    keep = torch.ones(V, dtype=torch.bool, device=z.device)
                    keep[cols] = False
                    part = part + rest * (math.log(rest) - (torch.logsumexp(zt[keep], 0) - lse))
            loss = loss + wd * T * T * part
        if labelled:
            loss = loss + wl * (torch.logsumexp(z[n], 0) - z[n, int(y[n])])
        on = bool(len(cols)) or labelled
        losses.append(loss if on else z.new_zeros(()))
        lses.append(lse.detach() if on else z.new_zeros(()))
        live.append(on)
    return torch.stack(losses), torch.stack(lses), torch.tensor(live, device=z.device)


def with_gradients(hidden, weight, loss_of, row_weight=None):
    """loss_of(z) -> (loss, lse, live) in float64.  Returns a dict of values and of bounds on the kernels' errors."""
    h, w = hidden.double(), weight.double()
    z = (h @ w.t()).requires_grad_(True)
    loss, lse, live = loss_of(z)
    rw = row_weight.double() if row_weight is not None else torch.full_like(loss, 1.0 / max(1, int(live.sum())))
    rw = torch.where(live, rw, 0.0)
    if loss.requires_grad:
        (loss * rw).sum().backward()
    dz = z.grad if z.grad is not None else torch.zeros_like(z)
    hz = torch.where(live[:, None], h, 0.0)            # rows that take no part do not enter the products
    out = {"loss": loss.detach(), "lse": lse.detach(), "grad_hidden": dz @ w, "grad_weight": dz.t() @ hz, "dz": dz, "live": live,
           "abs_h": (dz.abs() @ w.abs()), "abs_w": dz.abs().t() @ hz.abs()}
    # Logits: exact bf16 products added in fp32, one rounding or truncation (2^-23 of the magnitudes added so far) per
    # 16 products and one per step of the tree inside them.
    d, V, n = h.shape[1], w.shape[0], h.shape[0]
    size = float((hz.abs() @ w.abs().t()).max()) if n else 0.0
    out["e_z"] = size * (d / 16 + 6) * 2.0 ** -23
    # 2^x in fp32: the argument z log2(e) / T is rounded (2^-23 of it), the result is good to 2^-22
    top = float((z.detach().abs().masked_fill(~live[:, None], 0.0)).max()) if n else 0.0
    out["e_p"] = 2 * out["e_z"] + (top * 1.45 + 4) * 2.0 ** -22 + 2.0 ** -20
    out["steps_h"], out["steps_w"] = V / 16 + 40, n / 16 + 6
    return out


def check_rows(ref, loss, lse, scale=1.0, T=1.0):
    """scale: factor in front of the loss's logarithms (T^2 times weights)."""
    for name, got, f in (("loss", loss, 2 * scale), ("lse", lse, 1.0)):
        want = ref[name]
        lim = f * (2 * ref["e_z"] / min(T, 1.0) + ref["e_p"]) + 2.0 ** -22 * want.abs()
        d = (got.double() - want).abs()
        assert bool((d <= lim).all()), (name, float((d - lim).max()), float(d.max()))


def check_grads(ref, grad_hidden=None, grad_weight=None, small=0.0):
    """dL/dz is rounded to bf16 (unit roundoff 2^-8), or enters as two bf16 terms (2^-16) for fp32 weight gradients; then
    fp32 sums and the rounding of the result (2^-8 bf16, 2^-24 fp32).  `small`: extra absolute error of dL/dz per unit of row weight (cancelling terms)."""
    if grad_hidden is not None:
        lim = ref["abs_h"] * (2.0 ** -8 + ref["e_p"] + ref["steps_h"] * 2.0 ** -23) + 2.0 ** -8 * ref["grad_hidden"].abs() + 1e-30 + small
        d = (grad_hidden.double() - ref["grad_hidden"]).abs()
        assert bool((d <= lim).all()), ("grad_hidden", float((d - lim).max()), float(d.max()))
    if grad_weight is not None:
        f32 = grad_weight.dtype == torch.float32
        lim = ref["abs_w"] * ((2.0 ** -16 if f32 else 2.0 ** -8) + ref["e_p"] + 2 * ref["steps_w"] * 2.0 ** -23)
        lim = lim + (2.0 ** -23 if f32 else 2.0 ** -8) * ref["grad_weight"].abs() + 1e-30 + small
        d = (grad_weight.double() - ref["grad_weight"]).abs()
        assert bool((d <= lim).all()), ("grad_weight", float((d - lim).max()), float(d.max()))
