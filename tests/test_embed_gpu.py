"""Embedding lookup and its gradient against plain 64-bit forms."""
import math

import pytest
import torch

from tests import layers_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def embedding(*a, **kw):
    from paper_2609_20359_b200.embed import Embedding
    return Embedding(*a, device=DEV, **kw)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows(n, d, dtype, g, pad=0, shift=0, scale=1.0):
    """[n, d] with `pad` elements between rows, starting `shift` elements into its memory; NaN in what is not its own."""
    flat = torch.full((shift + n * (d + pad) + 16,), float("nan"), dtype=dtype, device=DEV)
    t = flat[shift:].as_strided((n, d), (d + pad, 1))
    t.copy_(scale * torch.randn(n, d, generator=g, device=DEV))
    return t, flat


def outside(flat, t):
    """What lies in flat beside t's elements."""
    own = torch.zeros(flat.shape, dtype=torch.bool, device=DEV)
    own.as_strided(t.shape, t.stride(), t.storage_offset() - flat.storage_offset()).fill_(True)
    return flat[~own]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("n,V,d,pad,shift,scale", [
    (1, 50257, 768, 0, 0, 1.0), (1, 5, 1, 0, 0, 1.0), (37, 1000, 767, 0, 0, 3.0), (64, 300, 1024, 8, 8, 0.5), (65, 300, 2048, 0, 1, 45.25),
    (9, 17, 1100, 4, 0, 1.0), (1000, 33, 36, 3, 5, -1.0), (5, 2, 65536, 0, 0, 1.0), (300, 128256, 8, 0, 0, 1.0), (4097, 91, 132, 4, 0, 1.0)])
def test_lookup(act, n, V, d, pad, shift, scale):
    g = gen(n + d)
    w, _ = rows(V, d, torch.bfloat16, g, pad, shift)
    out, flat = rows(n, d, TYPES[act], g, pad, shift)
    beside = outside(flat, out).clone()
    tok = torch.randint(0, V, (n,), generator=g, device=DEV)
    if n > 8:
        tok[3], tok[5], tok[7] = -100, V, -1
    e = embedding(n, V, d, act_dtype=act, grads=False)
    want = R.lookup(tok, w, scale, -100, TYPES[act])
    got = e.lookup(tok, w, scale=scale)
    assert got.is_contiguous() and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(got.isnan(), want.isnan())
    assert e.lookup(tok, w, out=out, scale=scale) is out
    assert torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0))
    assert torch.equal(outside(flat, out).isnan(), beside.isnan())
    # an ignored token inside the table, and tokens far outside
    tok[0] = 1 if V > 1 else 0
    if n > 8:
        tok[1], tok[2] = 2 ** 40, -2 ** 62
    got = e.lookup(tok, w, ignore_token=int(tok[0]))
    want = R.lookup(tok, w, 1.0, int(tok[0]), TYPES[act])
    assert bool((got[0] == 0).all()) and torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


def test_lookup_without_tokens():
    e = embedding(4, 10, 8)
    assert e.lookup(torch.empty(0, dtype=torch.int64, device=DEV), torch.zeros(10, 8, dtype=torch.bfloat16, device=DEV)).shape == (0, 8)


def tokens_of(kind, n, V, g):
    if kind == "random":
        return torch.randint(0, V, (n,), generator=g, device=DEV)
    if kind == "same":
        return torch.full((n,), V // 2, dtype=torch.int64, device=DEV)
    if kind == "few":
        return torch.randint(0, 3, (n,), generator=g, device=DEV) * ((V - 1) // 2)
    if kind == "text":                                                     # falling frequencies
        u = torch.rand(n, generator=g, device=DEV, dtype=torch.float64)
        return (torch.exp(u * math.log(V + 1)) - 1).long().clamp_(0, V - 1)
    if kind == "falling":
        return (V - 1 - torch.arange(n, device=DEV)) % V
    if kind == "ignored":
        return torch.full((n,), -100, dtype=torch.int64, device=DEV)
    if kind == "mixed":                                                    # half ignored, some outside
        t = torch.randint(0, V, (n,), generator=g, device=DEV)
        t[torch.rand(n, generator=g, device=DEV) < 0.5] = -100
        t[::7] = V
        t[3::11] = -2 ** 40
        return t
    raise ValueError(kind)


GRADS = [
    # n, V, d, tokens, pad, shift
    (1, 50257, 768, "random", 0, 0), (1, 1, 1, "same", 0, 0), (2, 3, 8, "same", 0, 0), (7, 1, 5, "same", 0, 0), (8, 2, 16, "few", 0, 0),
    (9, 1000, 33, "falling", 0, 0), (128, 5003, 768, "text", 0, 0), (129, 5003, 767, "text", 0, 0), (1000, 5003, 1000, "mixed", 0, 0),
    (1000, 400, 264, "ignored", 0, 0), (2048, 97, 300, "few", 4, 4), (4096, 1031, 256, "same", 0, 0), (4097, 1031, 128, "random", 8, 8),
    (5000, 128256, 64, "text", 0, 0), (16384, 511, 64, "few", 0, 0), (16385, 512, 72, "text", 0, 0), (33000, 513, 40, "mixed", 3, 1),
    (70000, 3, 24, "same", 0, 0), (131072, 40000, 8, "text", 0, 0), (131073, 40000, 8, "mixed", 0, 0), (300000, 70001, 9, "text", 0, 0),
    (256, 4001, 520, "text", 0, 0), (255, 9, 264, "few", 0, 0), (200, 3, 1000, "same", 0, 0), (257, 4001, 72, "mixed", 8, 8),
    (512, 1031, 77, "text", 0, 0), (511, 2, 96, "same", 0, 0), (300, 300000, 128, "random", 0, 0), (300, 300000, 16, "random", 0, 0), (50, 7, 65536, "random", 0, 0), (3000, 1 << 20, 8, "random", 0, 0), (200, 20000, 2048, "text", 0, 0)]


@pytest.mark.parametrize("act,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("n,V,d,kind,pad,shift", GRADS)
def test_grad(act, grad, n, V, d, kind, pad, shift):
    g = gen(n + d)
    dy, _ = rows(n, d, TYPES[act], g, pad, shift, 1e-3)
    gw, flat = rows(V, d, TYPES[grad], g, pad, shift)
    tok = tokens_of(kind, n, V, g)
    if kind in ("mixed", "ignored"):
        dy[(tok < 0) | (tok >= V)] = float("nan")                          # never read
    e = embedding(n, V, d, act_dtype=act, grad_dtype=grad)
    e.workspace.memory.fill_(255)
    gw.fill_(float("nan"))
    e.grad(tok, dy, gw, scale=1.7)
    R.check_embed_grad(gw, tok, dy, scale=1.7)
    assert bool(outside(flat, gw).isnan().all())
    first = gw.clone()
    e.grad(tok, dy, gw, scale=1.7)
    assert torch.equal(first, gw)                                          # the same bits every time
    base = torch.randn(V, d, generator=g, device=DEV).to(TYPES[grad])
    gw.copy_(base)
    e.grad(tok, dy, gw, scale=-0.3, accumulate=True)
    R.check_embed_grad(gw, tok, dy, scale=-0.3, old=base)
    assert bool(outside(flat, gw).isnan().all())


def test_grad_without_tokens():
    e = embedding(4, 10, 8, grad_dtype="f32")
    gw = torch.ones(10, 8, device=DEV)
    none, dy = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, 8, dtype=torch.bfloat16, device=DEV)
    e.grad(none, dy, gw, accumulate=True)
    assert bool((gw == 1).all())
    e.grad(none, dy, gw)
    assert bool((gw == 0).all())


def test_grad_of_a_smaller_call_and_of_every_length():
    """One workspace, calls of falling and rising size: nothing of an earlier call is left over."""
    V, d = 61, 24
    e = embedding(700, V, d, grad_dtype="f32")
    g = gen(5)
    gw = torch.empty(V, d, device=DEV)
    for n in list(range(1, 40)) + [700, 64, 65, 511, 512, 513, 3, 699]:
        tok, dy = tokens_of("text", n, V, g), rows(n, d, torch.bfloat16, g)[0]
        e.grad(tok, dy, gw)
        R.check_embed_grad(gw, tok, dy)


def test_grad_beyond_32_bits():
    """Rows of the gradient, and of what is summed, that start beyond 2^32 elements."""
    V, d, n = 66000, 65536, 5
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    g = gen(0)
    gw = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    gw[::997].fill_(5.0)
    tok = torch.tensor([V - 1, 0, V - 1, 65999, 65537], device=DEV)
    dy, _ = rows(n, d, torch.bfloat16, g)
    e = embedding(n, V, d)
    e.grad(tok, dy, gw)
    for v in (0, 65537, V - 1):
        want = dy[tok == v].double().sum(0)
        R.check("row", gw[v], want, R.U * 4 * dy[tok == v].double().abs().sum(0))
    assert int(torch.count_nonzero(gw[1:65537])) == 0 and int(torch.count_nonzero(gw[65538:V - 1])) == 0
    w = gw                                                                 # a table of as many bytes
    got = e.lookup(tok, w)
    assert torch.equal(got, w[tok])


def test_captured_and_replayed():
    V, d, n = 5000, 256, 600
    g = gen(1)
    e = embedding(n, V, d)
    tok, (dy, _) = tokens_of("text", n, V, g), rows(n, d, torch.bfloat16, g)
    w = torch.randn(V, d, generator=g, device=DEV).bfloat16()
    gw, out = torch.empty_like(w), torch.empty(n, d, dtype=torch.bfloat16, device=DEV)
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        e.grad(tok, dy, gw)
        e.lookup(tok, w, out=out)
    torch.cuda.current_stream().wait_stream(s)
    with torch.cuda.graph(graph):
        e.grad(tok, dy, gw)
        e.lookup(tok, w, out=out)
    for seed in (2, 3):
        h = gen(seed)
        tok.copy_(tokens_of("mixed", n, V, h))
        dy.copy_(torch.randn(n, d, generator=h, device=DEV))
        gw.fill_(float("nan"))
        graph.replay()
        R.check_embed_grad(gw, tok, dy)
        want = R.lookup(tok, w, 1.0, -100, torch.bfloat16)
        assert torch.equal(out.isnan(), want.isnan()) and torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0))
    del graph


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_on_another_stream(how):
    """The inputs are still being written when the call is made, on the stream that it is made for."""
    V, d, n = 5000, 512, 3000
    g = gen(1)
    tok, (dy, _) = tokens_of("text", n, V, g), rows(n, d, torch.bfloat16, g)
    w = torch.randn(V, d, generator=g, device=DEV).bfloat16()
    e = embedding(n, V, d)
    gw = torch.empty_like(w)
    late_tok, late_dy = torch.zeros_like(tok), torch.zeros_like(dy)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(50_000_000)
        late_tok.copy_(tok)
        late_dy.copy_(dy)
    kw = dict(stream=s if how == "stream" else s.cuda_stream) if how != "current" else {}
    with torch.cuda.stream(s if how == "current" else torch.cuda.default_stream()):
        e.grad(late_tok, late_dy, gw, **kw)
        out = e.lookup(late_tok, w, **kw)
    torch.cuda.synchronize()
    R.check_embed_grad(gw, tok, dy)
    assert torch.equal(out, w[tok])


def test_special_values():
    """Infinities, NaN and zeros of either sign go through as they are, and stay in their rows."""
    V, d = 20, 32
    e = embedding(64, V, d, grad_dtype="f32", act_dtype="f32")
    tok = torch.arange(64, device=DEV) % 16
    dy = torch.ones(64, d, device=DEV)
    dy[3] = float("inf")
    dy[4] = float("nan")
    dy[5], dy[21] = float("inf"), float("-inf")
    dy[6] = 3e38
    dy[22] = 3e38
    gw = torch.empty(V, d, device=DEV)
    e.grad(tok, dy, gw)
    want = torch.zeros(V, d, device=DEV).index_add_(0, tok, dy)
    assert torch.equal(gw.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))


def test_refusals():
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.embed import Embedding
    e = embedding(8, 100, 16)
    tok = torch.zeros(8, dtype=torch.int64, device=DEV)
    w = torch.zeros(100, 16, dtype=torch.bfloat16, device=DEV)
    dy = torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV)
    for bad in (lambda: e.lookup(tok.int(), w), lambda: e.lookup(tok[:, None], w), lambda: e.lookup(tok.cpu(), w),
                lambda: e.lookup(tok, w.float()), lambda: e.lookup(tok, w[:99]), lambda: e.lookup(tok, w.t()),
                lambda: e.lookup(tok, w, out=torch.empty(7, 16, dtype=torch.bfloat16, device=DEV)),
                lambda: e.grad(tok, dy.float(), w), lambda: e.grad(tok, dy[:7], w), lambda: e.grad(tok, dy, w.float()),
                lambda: e.grad(tok, dy[:1].expand(8, 16), w), lambda: e.grad(torch.zeros(16, dtype=torch.int64, device=DEV)[::2], dy, w),
                lambda: Embedding(8, 100, 16, act_dtype="f16"), lambda: Embedding(8, 100, 16, grad_dtype="bf8")):
        with pytest.raises(ValueError):
            bad()

    def refused(code, f, *a, **kw):
        with pytest.raises(fls.FlsError) as err:
            f(*a, **kw)
        assert err.value.code == code

    refused(fls.FLS_EINVAL, e.lookup, torch.zeros(9, dtype=torch.int64, device=DEV), w)
    refused(fls.FLS_EINVAL, e.lookup, tok, w, scale=math.nan)
    refused(fls.FLS_EINVAL, e.grad, tok, dy, w, scale=1e39)
    refused(fls.FLS_EINVAL, embedding(8, 100, 16, grads=False).grad, tok, dy, w)
    refused(fls.FLS_EPTR, e.lookup, tok, w, out=w[:8])
    refused(fls.FLS_EPTR, e.grad, tok, w[:8], w)
    refused(fls.FLS_EPTR, e.grad, tok, e.workspace.memory[:256].view(torch.bfloat16).view(8, 16), w)
    torch.cuda.synchronize()
