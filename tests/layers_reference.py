"""Plain 64-bit forms of the embedding and of the norms, and the error bounds the kernels are held to.

u = 2^-24 is half a step of fp32.  A sum of k terms in fp32, in any order whose longest chain has K additions, is off by at
most K u times the sum of the magnitudes (first order; the 1.01 below covers the rest).  Every output is rounded once more,
by at most half a step of its type."""
from __future__ import annotations

import torch

U = 2.0 ** -24
TINY = 1e-37                                         # below fp32's and bf16's normal numbers


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def check(name, got, want, lim):
    """lim: bound before the last rounding."""
    lim = 1.01 * lim + half_step(got.dtype) * (want.abs() + lim) + TINY
    d = (got.double() - want).abs()
    ok = (d <= lim) | (got.double() == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool(ok.all()), (name, float(torch.where(ok, 0.0, d - lim).max()), float(d.max()), int((~ok).sum()))


# ------------------------------------------------------------------------------------------------ embedding
def lookup(tokens, weight, scale, ignore, dtype):
    """To the bit: one fp32 product, one rounding."""
    V = weight.shape[0]
    ok = (tokens >= 0) & (tokens < V) & (tokens != ignore)
    out = (weight[tokens.clamp(0, V - 1)].float() * torch.tensor(scale, dtype=torch.float32, device=weight.device)).to(dtype)
    out[~ok] = float("nan")
    out[tokens == ignore] = 0
    return out


def embed_grad(tokens, grad_out, vocab, scale, ignore, old=None):
    """(gradient, sum of magnitudes, number of terms) of every row."""
    ok = (tokens >= 0) & (tokens < vocab) & (tokens != ignore)
    d = grad_out.shape[1]
    t, g = tokens[ok], grad_out[ok].double() * scale
    total = torch.zeros(vocab, d, dtype=torch.float64, device=grad_out.device)
    size, count = torch.zeros_like(total), torch.zeros(vocab, dtype=torch.float64, device=grad_out.device)
    total.index_add_(0, t, g)
    size.index_add_(0, t, g.abs())
    count.index_add_(0, t, torch.ones(len(t), dtype=torch.float64, device=grad_out.device))
    if old is not None:
        total += old.double()
    return total, size, count


def check_embed_grad(got, tokens, grad_out, scale=1.0, ignore=-100, old=None):
    want, size, count = embed_grad(tokens, grad_out, got.shape[0], scale, ignore, old)
    # a chain of at most `count` additions, scale as fp32 and its product, the addition to what was there
    lim = U * ((count[:, None] + 2) * size + want.abs() * (old is not None))
    check("grad_weight", got, want, lim)
    untouched = count == 0
    if old is None:
        assert bool((got[untouched] == 0).all())
    else:
        assert torch.equal(got[untouched].view(torch.uint8), old[untouched].view(torch.uint8))


# ------------------------------------------------------------------------------------------------ norms
def statistics(s, eps, rms):
    """(mean, rstd) of double rows."""
    mean = torch.zeros(s.shape[0], dtype=torch.float64, device=s.device) if rms else s.mean(1)
    var = (s - mean[:, None]).square().mean(1)
    return mean, 1.0 / torch.sqrt(var + eps)


def forward(s, weight, bias, eps, rms):
    mean, rstd = statistics(s, eps, rms)
    y = (s - mean[:, None]) * rstd[:, None]
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean, rstd


def check_forward(s, weight, bias, eps, rms, y, mean, rstd):
    """s: what is normalised, as the kernel saw it.  A thread adds up at most d / 32 values one by one (at least a warp works on
    a row), then trees join at most 2^10 of them: chains of K = d / 32 + 16."""
    d = s.shape[1]
    K = d / 32 + 16
    sd = s.double()
    want, m64, r64 = forward(sd, weight, bias, eps, rms)
    spread = (sd - m64[:, None]).square().mean(1).sqrt()
    if not rms:
        # the fp32 mean that is taken off first is K u mean|s| from the true one; what the second look sums is that much larger
        spread = spread + K * U * sd.abs().mean(1)
    centre = 3 * U * (sd - m64[:, None]).abs() + (0 if rms else 1) * (K + 4) * U * spread[:, None]
    # a relative error of var + eps halves in its root; the addition of eps, root, reciprocal: one rounding each
    rel = U * (0.5 * (K + 8) * (spread.square() * r64.square()) + 4)
    w = torch.ones(d, dtype=torch.float64, device=s.device) if weight is None else weight.double()
    xhat = (sd - m64[:, None]) * r64[:, None]
    lim = (xhat * w).abs() * (rel[:, None] + 3 * U) + w.abs() * r64[:, None] * centre + 2 * U * want.abs()
    if bias is not None:
        lim = lim + U * (xhat * w).abs()
    check("y", y, want, lim)
    if rstd is not None:
        check("rstd", rstd, r64, r64 * rel)
    if mean is not None:
        check("mean", mean, m64, 2 * U * m64.abs() + (K + 4) * U * spread)


def backward(x, weight, mean, rstd, grad_y, grad_total=None):
    """(grad_x, grad_weight, grad_bias) in 64 bits of the given statistics."""
    x, dy, r = x.double(), grad_y.double(), rstd.double()[:, None]
    xh = (x if mean is None else x - mean.double()[:, None]) * r
    g = dy if weight is None else dy * weight.double()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if mean is not None:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * r
    if grad_total is not None:
        dx = dx + grad_total.double()
    return dx, (dy * xh).sum(0), dy.sum(0)


def check_backward(x, weight, mean, rstd, grad_y, grad_total=None, grad_x=None, grad_weight=None, grad_bias=None, old_weight=None, old_bias=None):
    n, d = x.shape
    K = d / 32 + 16
    dx, dw, db = backward(x, weight, mean, rstd, grad_y, grad_total)
    xd, dy, r = x.double(), grad_y.double(), rstd.double()[:, None]
    xh = ((xd if mean is None else xd - mean.double()[:, None]) * r).abs()
    g = (dy if weight is None else dy * weight.double()).abs()
    if grad_x is not None:
        m1 = 0.0 if mean is None else g.mean(1, keepdim=True)
        m2 = (g * xh).mean(1, keepdim=True)
        lim = r * U * (6 * g + (K + 6) * m1 + (K + 12) * xh * m2) + 2 * U * dx.abs()
        check("grad_x", grad_x, dx, lim)
    # the product and xhat are rounded (four times in all); chains of at most n additions, and the one to what was there
    if grad_weight is not None:
        old = 0.0 if old_weight is None else old_weight.double()
        check("grad_weight", grad_weight, dw + old, U * ((n + 5) * (dy.abs() * xh).sum(0) + (dw + old).abs()))
    if grad_bias is not None:
        old = 0.0 if old_bias is None else old_bias.double()
        check("grad_bias", grad_bias, db + old, U * ((n + 1) * dy.abs().sum(0) + (db + old).abs()))
