"""The language-model head operators that are measured: cross entropy of a linear head without kept logits, distillation
from a teacher's top logits on the same head, and the selection of those top logits.

`run` with `own` false is the plain form in 32 bits; with `own` true it makes the calls a training program makes.
"""
import math

import torch

own = False

DEV = "cuda:0"
IGNORE = -100


# ------------------------------------------------------------------------------------------------ cases
def _head(name, op, rows, vocab, dim, **kw):
    c = dict(name=name, op=op, rows=rows, vocab=vocab, dim=dim, ignored=0.0, smoothing=0.0, z_loss=0.0, f32_grad=False,
             top=0, temperature=1.0, tail=False, distill_weight=0.0, label_weight=1.0)
    c.update(kw)
    return c


def listed():
    return [
        # one token's loss on a GPT-2-small-sized head: latency and one pass over the weight
        _head("xent_one_token", "xent", 1, 50257, 768),
        # perplexity of an evaluation batch on a Llama-3.2-1B-sized head
        _head("xent_eval_2048", "xent", 2048, 128256, 2048, ignored=0.05),
        # a small micro-batch of one group, bf16 gradient buffers
        _head("xent_step_128", "xent_step", 128, 50257, 768),
        # an odd batch, half of it prompt tokens without a label; fp32 gradient buffers, smoothing and z loss
        _head("xent_step_f32_1000", "xent_step", 1000, 50257, 768, ignored=0.45, smoothing=0.1, z_loss=1e-4, f32_grad=True),
        # one sequence on a head as wide as a Llama-3.1-8B block
        _head("xent_step_wide_1023", "xent_step", 1023, 128256, 4096),
        # a full micro-batch of four 2048-token sequences on the 1B-sized head
        _head("xent_step_8192", "xent_step", 8192, 128256, 2048),
        # scoring a few tokens against a teacher
        _head("distill_37", "distill", 37, 50257, 768, top=8, temperature=1.0, distill_weight=1.0, label_weight=0.0),
        # a distillation step at temperature 2 mixed with the labels, teacher list renormalised
        _head("distill_step_1024", "distill_step", 1024, 128256, 2048, top=64, temperature=2.0, distill_weight=0.5, label_weight=0.5),
        # a distillation step whose teacher gives its log sum exp: what is outside the list counts as one class
        _head("distill_step_tail_4096", "distill_step", 4096, 50257, 768, top=32, temperature=1.0, tail=True, distill_weight=1.0,
              label_weight=0.0, ignored=0.1),
        # a teacher's single token
        dict(name="top_one_token", op="top", rows=1, vocab=128256, top=64, temperature=1.0, f32_logits=False),
        # an odd batch of fp32 logits
        dict(name="top_f32_333", op="top", rows=333, vocab=50257, top=20, temperature=2.0, f32_logits=True),
        # a teacher's whole batch, bf16 logits
        dict(name="top_4096", op="top", rows=4096, vocab=128256, top=64, temperature=1.0, f32_logits=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["xent", "xent_step", "xent_step", "distill", "distill_step", "distill_step", "top"])
    vocab = _log_int(rng, 1000, 131072)
    if rng.random() < 0.5:
        vocab |= 1
    if op == "top":
        rows = _log_int(rng, 1, 4096)
        return dict(op="top", rows=rows, vocab=vocab, top=rng.randint(1, 128), temperature=rng.choice([1.0, 2.0, 4.0]),
                    f32_logits=rng.random() < 0.4)
    dim = 8 * _log_int(rng, 8, 512)
    rows = _log_int(rng, 1, 8192)
    most = 8192 * 128256 * 2048
    rows = max(1, min(rows, most // (2 * vocab * dim)))
    c = _head("", op, rows, vocab, dim, ignored=rng.choice([0.0, 0.1, 0.5]))
    del c["name"]
    if op.startswith("xent"):
        c.update(smoothing=rng.choice([0.0, 0.0, 0.1]), z_loss=rng.choice([0.0, 0.0, 1e-4]))
    else:
        c.update(top=rng.randint(1, 128), temperature=rng.choice([1.0, 2.0, 3.0]), tail=rng.random() < 0.4, distill_weight=0.7,
                 label_weight=rng.choice([0.0, 0.3]))
    c.update(f32_grad=op.endswith("step") and rng.random() < 0.25)
    return c


def work(case):
    n, v = case["rows"], case["vocab"]
    if case["op"] == "top":
        k = case["top"]
        return {"bytes": n * v * (4 if case["f32_logits"] else 2) + n * (8 * k + 4), "flops": 3 * n * v}
    d, k = case["dim"], case["top"]
    active = n * (1 - case["ignored"])
    by = 2 * n * d + 2 * v * d + 16 * n + 8 * n * k
    if not case["op"].endswith("step"):
        return {"bytes": by, "flops": 2 * active * v * d}
    return {"bytes": by + 2 * n * d + (4 if case["f32_grad"] else 2) * v * d, "flops": 6 * active * v * d}


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    def rand(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    n, v = case["rows"], case["vocab"]
    s = {"case": case}
    if case["op"] == "top":
        s["logits"] = (2.5 * randn(n, v)).to(torch.float32 if case["f32_logits"] else torch.bfloat16)
        if own:
            from paper_2609_20359_b200.head import TopLogits
            s["plan"] = TopLogits(n, v, case["top"], device=DEV)
        return s
    d, k = case["dim"], case["top"]
    # logits of about unit variance and a token that stands out by a few units, as a model in training has them
    s["weight"] = (randn(v, d) / math.sqrt(d)).to(torch.bfloat16)
    s["labels"] = torch.randint(0, v, (n,), generator=g, device=DEV)
    lift = 2.0 + 6.0 * rand(n, 1)
    s["hidden"] = (1.5 * randn(n, d) + lift * s["weight"][s["labels"]].float()).to(torch.bfloat16)
    out = rand(n) < case["ignored"]
    if k:
        # the teacher's list: the label's neighbourhood in no order of index, falling logits; a few rows have fewer entries
        gap = torch.randint(1, max(2, v // k), (n, k), generator=g, device=DEV)
        s["top_index"] = ((s["labels"][:, None] + torch.cumsum(gap, 1) - gap[:, :1]) % v).to(torch.int32)
        s["top_logit"] = 9.0 - torch.cumsum(1.2 * rand(n, k), 1) + 0.5 * rand(n, 1)
        short = (rand(n, 1) < 0.05) & (torch.arange(k, device=DEV)[None, :] >= (k + 1) // 2)
        s["top_index"][short | out[:, None]] = -1
        if case["tail"]:
            t = (s["top_logit"] / case["temperature"]).masked_fill(s["top_index"] < 0, -math.inf)
            s["teacher_lse"] = torch.logsumexp(t, 1) - torch.log1p(-0.02 - 0.2 * rand(n))
            s["teacher_lse"] = torch.where(out, torch.zeros_like(s["teacher_lse"]), s["teacher_lse"])
    s["labels"] = torch.where(out, torch.full_like(s["labels"], IGNORE), s["labels"])
    step = case["op"].endswith("step")
    if step:
        s["grad_hidden"] = torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
        s["grad_weight"] = torch.empty(v, d, dtype=torch.float32 if case["f32_grad"] else torch.bfloat16, device=DEV)
    if own:
        from paper_2609_20359_b200.head import Head
        s["plan"] = Head(n, v, d, top=k, grad_dtype="f32" if case["f32_grad"] else "bf16", grads=step, device=DEV)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    if c["op"] == "top":
        return _plain_top(s, c)
    z = s["hidden"].float() @ s["weight"].float().t()
    return _plain_xent(s, c, z) if c["op"].startswith("xent") else _plain_distill(s, c, z)


def _run_own(s, c):
    plan = s["plan"]
    if c["op"] == "top":
        value, index, lse = plan(s["logits"], temperature=c["temperature"])
        return {"value": value, "index": index, "lse": lse}
    if c["op"].startswith("xent"):
        opt = dict(ignore_label=IGNORE, label_smoothing=c["smoothing"], z_loss=c["z_loss"])
        if c["op"] == "xent":
            loss, lse = plan.xent(s["hidden"], s["weight"], s["labels"], **opt)
            return {"loss": loss, "lse": lse}
        loss, lse = plan.xent_step(s["hidden"], s["weight"], s["labels"], s["grad_hidden"], s["grad_weight"], **opt)
    else:
        opt = dict(labels=s["labels"] if c["label_weight"] else None, teacher_lse=s.get("teacher_lse"), ignore_label=IGNORE,
                   temperature=c["temperature"], distill_weight=c["distill_weight"], label_weight=c["label_weight"])
        if c["op"] == "distill":
            loss, lse = plan.distill(s["hidden"], s["weight"], s["top_index"], s["top_logit"], **opt)
            return {"loss": loss, "lse": lse}
        loss, lse = plan.distill_step(s["hidden"], s["weight"], s["top_index"], s["top_logit"], s["grad_hidden"], s["grad_weight"], **opt)
    return {"loss": loss, "lse": lse, "grad_hidden": s["grad_hidden"], "grad_weight": s["grad_weight"]}


def _plain_grads(s, dz, out):
    out["grad_hidden"] = (dz @ s["weight"].float()).to(torch.bfloat16)
    out["grad_weight"] = (dz.t() @ s["hidden"].float()).to(s["grad_weight"].dtype)
    return out


def _plain_xent(s, c, z):
    y, eps, zeta, v = s["labels"], c["smoothing"], c["z_loss"], c["vocab"]
    live = y != IGNORE
    at = y.clamp_min(0)[:, None]
    lse = torch.logsumexp(z, 1)
    loss = (1 - eps) * (lse - z.gather(1, at)[:, 0]) + zeta * lse * lse
    if eps:
        loss = loss + eps * (lse - z.mean(1))
    out = {"loss": torch.where(live, loss, 0.0), "lse": torch.where(live, lse, 0.0)}
    if c["op"] == "xent":
        return out
    w = torch.where(live, 1.0 / live.sum().clamp_min(1), 0.0)
    dz = torch.exp(z.sub_(lse[:, None]), out=z)
    dz.mul_((w * (1 + 2 * zeta * lse))[:, None])
    if eps:
        dz.sub_((w * (eps / v))[:, None])
    dz.scatter_add_(1, at, (-w * (1 - eps))[:, None])
    return _plain_grads(s, dz, out)


def _plain_distill(s, c, z):
    T, a, b = c["temperature"], c["distill_weight"], c["label_weight"]
    n, v = z.shape
    has = s["top_index"] >= 0
    idx = s["top_index"].clamp_min(0).long()
    taught = has.any(1)
    y = s["labels"]
    labelled = (y != IGNORE) if b else torch.zeros_like(taught)
    live = taught | labelled
    zt = z / T
    lse = torch.logsumexp(zt, 1)
    t = (s["top_logit"] / T).masked_fill(~has, -math.inf)
    norm = s["teacher_lse"] if c["tail"] else torch.logsumexp(t, 1)
    logq = torch.where(has, t - norm[:, None], 0.0)
    q = torch.where(has, torch.exp(logq), 0.0)
    logp = zt.gather(1, idx) - lse[:, None]
    kl = (q * (logq - logp)).sum(1)
    inside = torch.zeros(n, v + 1, dtype=torch.bool, device=z.device)
    inside.scatter_(1, torch.where(has, idx, v), True)
    inside = inside[:, :v]
    scale = torch.ones_like(kl)
    if c["tail"]:
        qt = (1 - q.sum(1)).clamp_min(0)
        logpt = torch.logsumexp(zt.masked_fill(inside, -math.inf), 1) - lse
        kl = kl + torch.where(qt > 0, qt * (torch.log(qt) - logpt), 0.0)
        scale = 1 - qt * torch.exp(-logpt)
    loss = torch.where(taught, a * T * T * kl, 0.0)
    if b:
        lse1 = torch.logsumexp(z, 1)
        ce = lse1 - z.gather(1, y.clamp_min(0)[:, None])[:, 0]
        loss = loss + torch.where(labelled, b * ce, 0.0)
    out = {"loss": loss, "lse": torch.where(live, lse, 0.0)}
    if c["op"] == "distill":
        return out
    w = 1.0 / live.sum().clamp_min(1)
    at_rows = torch.where(taught, a * T * w, 0.0)
    p = torch.exp(zt.sub_(lse[:, None]), out=zt)
    dz = p.mul_(torch.where(inside, 1.0, scale[:, None]) if c["tail"] else 1.0).mul_(at_rows[:, None])
    dz.scatter_add_(1, idx, -q * at_rows[:, None])
    if b:
        bw = torch.where(labelled, b * w, 0.0)
        dz.add_(torch.exp(z - lse1[:, None]).mul_(bw[:, None]))
        dz.scatter_add_(1, y.clamp_min(0)[:, None], -bw[:, None])
    return _plain_grads(s, dz, out)


def _plain_top(s, c):
    z = s["logits"].float()
    value, index = torch.sort(z, dim=1, descending=True, stable=True)
    k = c["top"]
    return {"value": value[:, :k].contiguous(), "index": index[:, :k].to(torch.int32), "lse": torch.logsumexp(z / c["temperature"], 1)}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """From the definitions in 64 bits, the vocabulary taken in slices: sums first, then the probabilities slice by slice."""
    s = prepare(case, seed)
    c, v = case, case["vocab"]
    if c["op"] == "top":
        z = s["logits"]
        k = c["top"]
        parts = []
        for lo in range(0, z.shape[0], 256):
            x = z[lo: lo + 256].double()
            order = torch.argsort(-x, dim=1, stable=True)[:, :k]
            m = x.max(1).values
            lse = m / c["temperature"] + torch.log(torch.exp((x - m[:, None]) / c["temperature"]).sum(1))
            parts.append((x.gather(1, order), order.to(torch.int32), lse))
        value, index, lse = (torch.cat(x) for x in zip(*parts))
        return {"value": value, "index": index, "lse": lse}
    h, W = s["hidden"].double(), s["weight"]
    n, y = c["rows"], s["labels"]
    step = 16384
    lows = list(range(0, v, step))
    every = torch.arange(n, device=DEV)

    def logits(lo):
        return h @ W[lo: lo + step].double().t()

    def log_sum(T, drop=None):
        m = torch.full((n,), -math.inf, dtype=torch.float64, device=DEV)
        a = torch.zeros(n, dtype=torch.float64, device=DEV)
        total = torch.zeros_like(a)
        for lo in lows:
            x = logits(lo)
            total += x.sum(1)
            x = x / T
            if drop is not None:
                x[drop(lo, x.shape[1])] = -math.inf
            new = torch.maximum(m, x.max(1).values)
            a = a * torch.exp(m - new) + torch.exp(x - new[:, None]).sum(1)
            m = new
        return m + torch.log(a), total / v

    def at(cols):  # logits at given columns, -1 read as 0
        return torch.stack([(h * W[cols[:, j].clamp_min(0).long()].double()).sum(1) for j in range(cols.shape[1])], 1)

    def gradients(of_slice):
        dh = torch.zeros(n, c["dim"], dtype=torch.float64, device=DEV)
        dw = torch.empty(v, c["dim"], dtype=torch.float64 if c["f32_grad"] else torch.float32, device=DEV)
        for lo in lows:
            dz = of_slice(lo, logits(lo))
            dh += dz @ W[lo: lo + step].double()
            dw[lo: lo + step] = (dz.t() @ h).to(dw.dtype)
        return dh, dw

    def put(dz, lo, rows, cols, val):
        ok = (cols >= lo) & (cols < lo + dz.shape[1])
        dz.index_put_((rows[ok], cols[ok].long() - lo), val[ok], accumulate=True)

    if c["op"].startswith("xent"):
        eps, zeta = c["smoothing"], c["z_loss"]
        live = y >= 0
        lse, mean = log_sum(1.0)
        ce = lse - at(y[:, None])[:, 0]
        loss = (1 - eps) * ce + eps * (lse - mean) + zeta * lse ** 2
        out = {"loss": loss * live, "lse": lse * live}
        if c["op"] == "xent":
            return out
        w = live.double() / max(1, int(live.sum()))

        def of_slice(lo, x):
            dz = torch.exp(x - lse[:, None]) * ((1 + 2 * zeta * lse) * w)[:, None] - (eps / v) * w[:, None]
            put(dz, lo, every, y, -(1 - eps) * w)
            return dz
    else:
        T, a, b = c["temperature"], c["distill_weight"], c["label_weight"]
        cols = s["top_index"]
        has = cols >= 0
        taught = has.any(1)
        labelled = (y >= 0) & bool(b)
        rows = every[:, None].expand_as(cols)

        def listed_in(lo, width):
            ok = (cols >= lo) & (cols < lo + width)
            mark = torch.zeros(n, width, dtype=torch.bool, device=DEV)
            mark[rows[ok], cols[ok].long() - lo] = True
            return mark

        lse, _ = log_sum(T)
        t = s["top_logit"].double() / T
        top = torch.where(has, t, -math.inf).max(1, keepdim=True).values.nan_to_num(neginf=0.0)
        norm = s["teacher_lse"].double() if c["tail"] else (top[:, 0] + torch.log((torch.exp(t - top) * has).sum(1)))
        norm = torch.where(taught, norm, 0.0)
        logq = (t - norm[:, None]) * has
        q = torch.exp(logq) * has
        kl = (q * (logq - (at(cols) / T - lse[:, None]))).sum(1)
        damp = torch.ones_like(kl)
        if c["tail"]:
            qt = (1 - q.sum(1)).clamp_min(0)
            rest, _ = log_sum(T, listed_in)
            kl = kl + torch.where(qt > 0, qt * (torch.log(qt) - (rest - lse)), 0.0)
            damp = 1 - qt * torch.exp(lse - rest)
        loss = a * T * T * kl * taught
        if b:
            lse1, _ = log_sum(1.0)
            loss = loss + b * (lse1 - at(y[:, None])[:, 0]) * labelled
        live = taught | labelled
        out = {"loss": loss, "lse": lse * live}
        if c["op"] == "distill":
            return out
        w = 1.0 / max(1, int(live.sum()))

        def of_slice(lo, x):
            p = torch.exp(x / T - lse[:, None])
            if c["tail"]:
                p = torch.where(listed_in(lo, x.shape[1]), p, p * damp[:, None])
            dz = p * (a * T * w * taught.double())[:, None]
            put(dz, lo, rows[has], cols[has], -a * T * w * q[has])
            if b:
                dz += torch.exp(x - lse1[:, None]) * (b * w * labelled.double())[:, None]
                put(dz, lo, every[labelled], y[labelled], torch.full((int(labelled.sum()),), -b * w, dtype=torch.float64, device=DEV))
            return dz
    out["grad_hidden"], out["grad_weight"] = gradients(of_slice)
    return out
