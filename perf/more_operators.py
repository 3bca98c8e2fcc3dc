"""The operators around the head that are measured: embedding lookup and its gradient, and the norm (layer norm and root mean
square norm, with the residual addition before it) and its gradient.

`run` with `own` false is the plain form in 32 bits; with `own` true it makes the calls a training or serving program makes.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
IGNORE = -100
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ cases
def _embed(name, op, tokens, vocab, dim, **kw):
    c = dict(name=name, op=op, tokens=tokens, vocab=vocab, dim=dim, act="bf16", grad="bf16", ignored=0.0, scaled=False, micro=1)
    c.update(kw)
    return c


def _norm(name, op, rows, dim, **kw):
    c = dict(name=name, op=op, rows=rows, dim=dim, kind="layer", x="bf16", y="bf16", weight="bf16", grad="bf16", bias=False,
             residual=False, stats=True)
    c.update(kw)
    return c


def listed():
    return [
        # the next token of one stream on a GPT-2-small-sized table: latency
        _embed("lookup_one_token", "lookup", 1, 50257, 768),
        # an odd, padded batch into an fp32 residual stream
        _embed("lookup_f32_1000", "lookup", 1000, 50257, 768, act="f32", ignored=0.3),
        # a micro-batch of eight 2048-token sequences on a Llama-3.2-1B-sized table, scaled as some models do
        _embed("lookup_16384", "lookup", 16384, 128256, 2048, scaled=True),
        # a small micro-batch of one replica, the whole gradient unit written
        _embed("embed_grad_128", "embed_grad", 128, 50257, 768),
        # two micro-batches of 4096 tokens into the same bf16 gradient unit: written by the first, added to by the second
        _embed("embed_grad_two_4096", "embed_grad", 8192, 50257, 768, micro=2),
        # an odd, padded batch on the 1B-sized table, fp32 gradient buffers
        _embed("embed_grad_f32_8191", "embed_grad", 8191, 128256, 2048, act="bf16", grad="f32", ignored=0.1),
        # one token of one stream in front of a block: residual added, nothing kept for a backward pass
        _norm("norm_one_token", "norm", 1, 2048, kind="rms", residual=True, stats=False),
        # an odd batch of an fp32 residual stream, GPT-2-small-sized, with bias
        _norm("norm_f32_1000", "norm", 1000, 768, x="f32", bias=True),
        # a micro-batch of the 1B-sized model, residual added
        _norm("norm_16384", "norm", 16384, 2048, kind="rms", residual=True),
        # a small micro-batch, GPT-2-small-sized
        _norm("norm_grad_128", "norm_grad", 128, 768, bias=True),
        # one sequence of a model as wide as a Llama-3.1-8B block, the residual's gradient added
        _norm("norm_grad_1023", "norm_grad", 1023, 4096, kind="rms", residual=True),
        # sixteen 2048-token sequences, fp32 residual stream and fp32 gradient buffers
        _norm("norm_grad_f32_32768", "norm_grad", 32768, 768, x="f32", weight="f32", grad="f32", bias=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["lookup", "embed_grad", "embed_grad", "norm", "norm_grad", "norm_grad"])
    dim = 8 * _log_int(rng, 8, 512)
    if rng.random() < 0.15:
        dim -= rng.randint(1, 7)
    rows = max(1, min(_log_int(rng, 1, 65536), 16384 * 2048 // dim))
    if op in ("lookup", "embed_grad"):
        vocab = _log_int(rng, 1000, 131072)
        grad = "f32" if rng.random() < 0.3 else "bf16"
        vocab = min(vocab, 128256 * 2048 // dim)
        micro = 2 if op == "embed_grad" and rows > 1 and rng.random() < 0.3 else 1
        c = _embed("", op, rows, vocab, dim, act=rng.choice(["bf16", "bf16", "f32"]), grad=grad, ignored=rng.choice([0.0, 0.0, 0.2]),
                   scaled=rng.random() < 0.3, micro=micro)
    else:
        c = _norm("", op, rows, dim, kind=rng.choice(["layer", "rms"]), x=rng.choice(["bf16", "bf16", "f32"]),
                  y=rng.choice(["bf16", "bf16", "f32"]), weight=rng.choice(["bf16", "f32"]), grad=rng.choice(["bf16", "f32"]),
                  bias=rng.random() < 0.5, residual=rng.random() < 0.5, stats=op == "norm_grad" or rng.random() < 0.7)
    del c["name"]
    return c


def _distinct(case):
    """Expected number of different tokens (of the distribution in _tokens) among those that count."""
    v = case["vocab"]
    k = np.arange(1, v + 1, dtype=np.float64)
    p = np.log1p(1 / k) / math.log(v + 1)
    return float(-np.expm1(case["tokens"] * (1 - case["ignored"]) * np.log1p(-p)).sum()) if v > 1 else 1.0


def work(case):
    if case["op"] in ("lookup", "embed_grad"):
        n, d, v = case["tokens"], case["dim"], case["vocab"]
        rows = n * d * SIZE[case["act"]]
        if case["op"] == "lookup":
            return {"bytes": 8 * n + 2 * d * _distinct(case) + rows, "flops": n * d}
        g = SIZE[case["grad"]]
        again = 2 * g * d * _distinct(dict(case, tokens=n // 2)) if case["micro"] == 2 else 0
        return {"bytes": 8 * n + rows * (1 - case["ignored"]) + g * v * d + again, "flops": n * d}
    n, d = case["rows"], case["dim"]
    x, y, w = SIZE[case["x"]], SIZE[case["y"]], SIZE[case["weight"]]
    if case["op"] == "norm":
        stats = n * (8 if case["kind"] == "layer" else 4) if case["stats"] else 0
        return {"bytes": n * d * (x + y + (2 * x if case["residual"] else 0)) + d * w * (2 if case["bias"] else 1) + stats, "flops": 8 * n * d}
    stats = n * (8 if case["kind"] == "layer" else 4)
    return {"bytes": n * d * (2 * x + y + (x if case["residual"] else 0)) + d * w + d * SIZE[case["grad"]] * (2 if case["bias"] else 1) + stats,
            "flops": 14 * n * d}


# ------------------------------------------------------------------------------------------------ inputs
def _tokens(n, vocab, ignored, g):
    """Tokens as text has them: the k-th most frequent one about k times rarer than the first, those spread over the table."""
    u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)) - 1).long().clamp_(0, vocab - 1)
    step = 7919 if math.gcd(7919, vocab) == 1 else 1
    tok = (rank * step + 11) % vocab
    if ignored:
        tok[torch.rand(n, generator=g, device=DEV) < ignored] = IGNORE
    return tok


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = {"case": case}
    d = case["dim"]
    if case["op"] in ("lookup", "embed_grad"):
        n, v, act = case["tokens"], case["vocab"], TYPES[case["act"]]
        s["tokens"] = _tokens(n, v, case["ignored"], g)
        s["scale"] = math.sqrt(d) if case["scaled"] else 1.0
        if case["op"] == "lookup":
            s["weight"] = (0.02 * randn(v, d)).to(torch.bfloat16)
        else:
            s["grad_out"] = (1e-3 * randn(n, d)).to(act)
            s["grad_weight"] = torch.empty(v, d, dtype=TYPES[case["grad"]], device=DEV)
        if own:
            from paper_2609_20359_b200.embed import Embedding
            s["plan"] = Embedding(n, v, d, act_dtype=case["act"], grad_dtype=case["grad"], grads=case["op"] == "embed_grad", device=DEV)
        return s
    n = case["rows"]
    xt, yt, wt = TYPES[case["x"]], TYPES[case["y"]], TYPES[case["weight"]]
    # a residual stream: off centre, a few channels that stand out, rows of different size
    channel = 0.2 * randn(d) + torch.where(torch.rand(d, generator=g, device=DEV) < 0.01, 8.0, 0.0)
    x = (randn(n, d) + channel) * torch.exp(0.5 * randn(n, 1))
    s["x"] = x.to(xt)
    s["weight"] = (1.0 + 0.3 * randn(d)).to(wt)
    s["bias"] = (0.1 * randn(d)).to(wt) if case["bias"] else None
    if case["op"] == "norm":
        s["residual"] = randn(n, d).to(xt) if case["residual"] else None
    else:
        s["grad_y"] = (1e-3 * randn(n, d)).to(yt)
        s["grad_total"] = (1e-3 * randn(n, d)).to(xt) if case["residual"] else None
        # kept by the forward pass
        x = s["x"]
        mean = x.mean(1, dtype=torch.float64) if case["kind"] == "layer" else torch.zeros(n, dtype=torch.float64, device=DEV)
        var = torch.cat([(p.double() - m[:, None]).square().mean(1) for p, m in zip(x.split(4096), mean.split(4096))])
        s["mean"] = mean.float() if case["kind"] == "layer" else None
        s["rstd"] = (var + EPS).rsqrt().float()
    if own:
        from paper_2609_20359_b200.norm import Norm
        s["plan"] = Norm(n, d, kind=case["kind"], eps=EPS, x_dtype=case["x"], y_dtype=case["y"], weight_dtype=case["weight"],
                         grad_dtype=case["grad"], grads=case["op"] == "norm_grad", device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"lookup": _plain_lookup, "embed_grad": _plain_embed_grad, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[c["op"]](s, c)


def _run_own(s, c):
    plan = s["plan"]
    if c["op"] == "lookup":
        return {"out": plan.lookup(s["tokens"], s["weight"], scale=s["scale"], ignore_token=IGNORE)}
    if c["op"] == "embed_grad":
        if c["micro"] == 1:
            plan.grad(s["tokens"], s["grad_out"], s["grad_weight"], scale=s["scale"], ignore_token=IGNORE)
        else:
            half = c["tokens"] // 2
            plan.grad(s["tokens"][:half], s["grad_out"][:half], s["grad_weight"], scale=s["scale"], ignore_token=IGNORE)
            plan.grad(s["tokens"][half:], s["grad_out"][half:], s["grad_weight"], scale=s["scale"], ignore_token=IGNORE, accumulate=True)
        return {"grad_weight": s["grad_weight"]}
    if c["op"] == "norm":
        out = {}
        if c["residual"]:
            out["y"], out["total"], mean, rstd = plan.add_forward(s["x"], s["residual"], s["weight"], s["bias"], stats=c["stats"])
        else:
            out["y"], mean, rstd = plan.forward(s["x"], s["weight"], s["bias"], stats=c["stats"])
        if mean is not None:
            out["mean"] = mean
        if rstd is not None:
            out["rstd"] = rstd
        return out
    dw = torch.empty(c["dim"], dtype=TYPES[c["grad"]], device=DEV)
    db = torch.empty_like(dw) if c["bias"] else None
    dx = plan.backward(s["x"], s["weight"], s["mean"], s["rstd"], s["grad_y"], grad_weight=dw, grad_bias=db, grad_total=s["grad_total"])
    out = {"grad_x": dx, "grad_weight": dw}
    if db is not None:
        out["grad_bias"] = db
    return out


def _plain_lookup(s, c):
    t = s["tokens"]
    rows = s["weight"][t.clamp_min(0)].float() * s["scale"]
    return {"out": rows.masked_fill_((t == IGNORE)[:, None], 0.0).to(TYPES[c["act"]])}


def _plain_embed_grad(s, c):
    t, d = s["tokens"], s["grad_out"]
    total = torch.zeros(c["vocab"], c["dim"], device=DEV)
    live = t != IGNORE
    total.index_add_(0, t.clamp_min(0), torch.where(live[:, None], d.float(), 0.0))
    s["grad_weight"].copy_(total.mul_(s["scale"]))
    return {"grad_weight": s["grad_weight"]}


def _plain_norm(s, c):
    out = {}
    x = s["x"]
    if c["residual"]:
        x = out["total"] = (x.float() + s["residual"].float()).to(x.dtype)
    x = x.float()
    if c["kind"] == "layer":
        mean = x.mean(1)
        x = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((x * x).mean(1) + EPS)
    y = x * rstd[:, None] * s["weight"].float()
    if c["bias"]:
        y = y + s["bias"].float()
    out["y"] = y.to(TYPES[c["y"]])
    if c["stats"]:
        out["rstd"] = rstd
        if c["kind"] == "layer":
            out["mean"] = mean
    return out


def _plain_norm_grad(s, c):
    x, dy, rstd = s["x"].float(), s["grad_y"].float(), s["rstd"][:, None]
    xhat = ((x - s["mean"][:, None]) if c["kind"] == "layer" else x) * rstd
    out = {"grad_weight": (dy * xhat).sum(0).to(TYPES[c["grad"]])}
    if c["bias"]:
        out["grad_bias"] = dy.sum(0).to(TYPES[c["grad"]])
    g = dy * s["weight"].float()
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if c["kind"] == "layer":
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd
    if c["residual"]:
        dx = dx + s["grad_total"].float()
    out["grad_x"] = dx.to(TYPES[c["x"]])
    return out


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """From the definitions in 64 bits: one-hot sums token by token where they are, statistics and gradients row by row."""
    s = prepare(case, seed)
    c = case
    if c["op"] == "lookup":
        t = s["tokens"]
        out = torch.zeros(c["tokens"], c["dim"], dtype=torch.float64, device=DEV)
        at = torch.nonzero(t >= 0)[:, 0]
        out[at] = s["weight"].double()[t[at]] * s["scale"]
        return {"out": out}
    if c["op"] == "embed_grad":
        # sorted tokens, running sums in 64 bits, differences at the ends of each token's stretch
        t = s["tokens"]
        order = torch.argsort(t, stable=True)
        order = order[t[order] >= 0]
        which, count = torch.unique_consecutive(t[order], return_counts=True)
        ends = torch.cumsum(count, 0)
        total = torch.zeros(c["vocab"], c["dim"], dtype=torch.float64 if c["grad"] == "f32" else torch.float32, device=DEV)
        for lo in range(0, c["dim"], 512):
            run_sum = torch.cumsum(s["grad_out"][:, lo: lo + 512].double()[order], 0)
            upto = run_sum[ends - 1]
            upto[1:] -= run_sum[ends[:-1] - 1]
            total[which, lo: lo + 512] = (upto * s["scale"]).to(total.dtype)
        return {"grad_weight": total}
    n, d, layer = c["rows"], c["dim"], c["kind"] == "layer"
    w = s["weight"].double()
    step = max(1, (64 << 20) // (8 * d))
    if c["op"] == "norm":
        parts = {"y": [], "rstd": [], "mean": [], "total": []}
        for lo in range(0, n, step):
            x = s["x"][lo: lo + step].double()
            if c["residual"]:
                x = x + s["residual"][lo: lo + step].double()
                parts["total"].append(x)
                x = x.to(TYPES[c["x"]]).double()               # what is normalised is what is returned
            var, mean = torch.var_mean(x, 1, correction=0)
            if not layer:
                var, mean = torch.linalg.vector_norm(x, dim=1).square() / d, torch.zeros_like(mean)
            r = (var + EPS) ** -0.5
            y = torch.einsum("nd,n,d->nd", x - mean[:, None], r, w)
            parts["y"].append(y + s["bias"].double() if c["bias"] else y)
            parts["rstd"].append(r)
            parts["mean"].append(mean)
        keep = ["y"] + (["total"] if c["residual"] else []) + (["rstd"] + (["mean"] if layer else []) if c["stats"] else [])
        return {k: torch.cat(parts[k]) for k in keep}
    dw = torch.zeros(d, dtype=torch.float64, device=DEV)
    db = torch.zeros_like(dw)
    dx = []
    for lo in range(0, n, step):
        at = slice(lo, lo + step)
        x, dy, r = s["x"][at].double(), s["grad_y"][at].double(), s["rstd"][at].double()
        xc = x - s["mean"][at].double()[:, None] if layer else x
        dw += torch.einsum("nd,nd,n->d", dy, xc, r)
        db += dy.sum(0)
        # d/dx of (x - mean) * rstd, the projection off the row (and off its mean)
        along = torch.einsum("nd,nd,d->n", dy, xc, w) * r ** 3 / d
        part = r[:, None] * w * dy - along[:, None] * xc
        if layer:
            part = part - ((dy @ w) * r / d)[:, None]
        dx.append(part + s["grad_total"][at].double() if c["residual"] else part)
    out = {"grad_weight": dw, "grad_x": torch.cat(dx)}
    if c["bias"]:
        out["grad_bias"] = db
    return out
