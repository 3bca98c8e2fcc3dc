"""CPU-side checks of the embedding and the norms: sizes, structures, refusals and launches on a CUDA runtime that only writes
them down, and the reference itself."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from tests import fake_cuda
from tests import layers_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def fls():
    from paper_2609_20359_b200 import build
    build.build()
    import paper_2609_20359_b200._binding as b
    return b


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fake_cuda.build(tmp_path_factory.mktemp("fake"))


def test_struct_layouts_match_the_header(fls, tmp_path):
    names = {n: getattr(fls, n) for n in ("fls_embed_desc", "fls_embed_layout", "fls_embed_io", "fls_norm_desc", "fls_norm_layout",
                                          "fls_norm_io", "fls_norm_grad_io")}
    body = "".join(f'  printf("%zu ", sizeof({n}));\n' + "".join(f'  printf("%zu ", offsetof({n}, {f[0]}));\n' for f in t._fields_)
                   for n, t in names.items())
    src = tmp_path / "s.c"
    src.write_text('#include "fls.h"\n#include <stddef.h>\n#include <stdio.h>\nint main(void) {\n' + body + "  return 0;\n}\n")
    exe = tmp_path / "s"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for t in names.values():
        want += [C.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want


def test_star_import_has_every_entry_point(fls):
    names = {}
    exec("from paper_2609_20359_b200._binding import *", names)
    assert [n for n in fls.EXPORTS if n not in names] == []
    assert {"fls_embed_grad", "fls_norm_backward"} <= set(fls.EXPORTS)


@pytest.mark.parametrize("kw", [dict(vocab=0), dict(vocab=(1 << 30) + 1), dict(dim=0), dict(dim=65537), dict(max_tokens=(1 << 24) + 1),
                                dict(act_dtype=2), dict(grad_dtype=7)])
def test_embed_create_refuses(fls, kw):
    with pytest.raises(fls.FlsError) as e:
        fls.fls_embed_create(**{**dict(max_tokens=16, vocab=1000, dim=64), **kw})
    assert e.value.code == fls.FLS_EINVAL and str(e.value)


@pytest.mark.parametrize("kw", [dict(dim=0), dict(dim=65537), dict(max_rows=(1 << 24) + 1), dict(kind=2), dict(x_dtype=2), dict(y_dtype=3),
                                dict(weight_dtype=2), dict(grad_dtype=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_norm_create_refuses(fls, kw):
    with pytest.raises(fls.FlsError) as e:
        fls.fls_norm_create(**{**dict(max_rows=16, dim=64), **kw})
    assert e.value.code == fls.FLS_EINVAL and str(e.value)


def test_null_arguments(fls):
    out = C.c_void_p()
    for kind in ("embed", "norm"):
        call = lambda n, *a: getattr(fls.lib, f"fls_{kind}_{n}")(*a)  # noqa: E731
        assert call("create", None, C.byref(out)) == fls.FLS_EINVAL
        assert call("query", None, None) == fls.FLS_EINVAL
        assert call("get_launch_count", None, None) == fls.FLS_EINVAL
        assert call("destroy", None) == fls.FLS_OK
    assert fls.lib.fls_embed_lookup(None, None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_embed_grad(None, None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_norm_forward(None, None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_norm_backward(None, None, None) == fls.FLS_EINVAL


BUFFERS = """
def at(i, d=0):
    return (d << 44) + (i + 1 << 40)

def io(kind, names, **kw):
    t = kind()
    for i, n in enumerate(names):
        setattr(t, n, at(i))
    for k, v in kw.items():
        setattr(t, k, v)
    return t

EMBED = ["token", "weight", "out", "grad_out", "grad_weight", "workspace"]
FORWARD = ["x", "residual", "weight", "bias", "y", "total", "mean", "rstd"]
BACKWARD = ["x", "weight", "mean", "rstd", "grad_y", "grad_total", "grad_x", "grad_weight", "grad_bias", "workspace"]

def embed_io(**kw):
    return io(fls.fls_embed_io, EMBED, **{**dict(tokens=4, ignore_token=-100, scale=1.0, workspace_bytes=1 << 30), **kw})

def forward_io(**kw):
    return io(fls.fls_norm_io, FORWARD, **{**dict(rows=4), **kw})

def backward_io(**kw):
    return io(fls.fls_norm_grad_io, BACKWARD, **{**dict(rows=4, workspace_bytes=1 << 30), **kw})
"""


def test_calls_refuse(fake):
    """Each call with one thing wrong: its code, and nothing launched."""
    got = fake_cuda.run(fake, BUFFERS + """
fake.fake_reset(0)
e = fls.fls_embed_create(16, 1000, 64)
n, rms = fls.fls_norm_create(16, 64), fls.fls_norm_create(16, 64, fls.FLS_NORM_RMS)
I, P, A, S = fls.FLS_EINVAL, fls.FLS_EPTR, fls.FLS_EALIGN, fls.FLS_ESIZE
big = 1 << 31
result = []
def want(c, f, *a):
    result.append([c, code(f, *a, stream=0), fake.fake_launches()])
both = [(I, dict(tokens=17)), (I, dict(reserved=1)), (I, dict(accumulate=2)), (I, dict(scale=float("nan"))), (I, dict(scale=1e39)),
        (I, dict(weight_stride=63)), (I, dict(out_stride=big)), (I, dict(grad_out_stride=1)), (I, dict(grad_weight_stride=big)),
        (A, dict(token=at(0) + 4)), (P, dict(token=0)), (P, dict(token=at(0, 15))), (P, dict(token=at(0, 1)))]
for c, kw in both + [(A, dict(weight=at(1) + 1)), (A, dict(out=at(2) + 1)), (P, dict(out=0)), (P, dict(weight=0)), (P, dict(out=at(1))),
                     (P, dict(out=at(0, 3)))]:
    want(c, fls.fls_embed_lookup, e, embed_io(**kw))
for c, kw in both + [(A, dict(grad_out=at(3) + 1)), (A, dict(grad_weight=at(4) + 1)), (A, dict(workspace=at(5) + 128)),
                     (S, dict(workspace_bytes=100)), (P, dict(workspace=0)), (P, dict(grad_weight=0)), (P, dict(grad_out=0)),
                     (P, dict(grad_weight=at(3))), (P, dict(workspace=at(4) + 256)), (P, dict(grad_weight=at(4, 2)))]:
    want(c, fls.fls_embed_grad, e, embed_io(**kw))
want(I, fls.fls_embed_grad, fls.fls_embed_create(16, 1000, 64, False), embed_io())
for c, kw in [(I, dict(rows=17)), (I, dict(reserved=1)), (I, dict(residual=0)), (I, dict(total=0)), (I, dict(x_stride=63)),
              (I, dict(residual_stride=big)), (I, dict(y_stride=1)), (I, dict(total_stride=big)), (P, dict(x=0)), (P, dict(y=0)), (P, dict(y=at(0))),
              (P, dict(y=at(5))), (P, dict(total=at(0), total_stride=65)), (P, dict(mean=at(7))), (P, dict(y=at(4, 15))), (P, dict(x=at(0, 1))),
              (A, dict(x=at(0) + 1)), (A, dict(mean=at(6) + 2)), (A, dict(weight=at(2) + 1)), (P, dict(y=at(2)))]:
    want(c, fls.fls_norm_forward, n, forward_io(**kw))
want(I, fls.fls_norm_forward, rms, forward_io())                       # has no mean
for c, kw in [(I, dict(rows=17)), (I, dict(reserved=1)), (I, dict(accumulate=2)), (I, dict(grad_x=0)), (I, dict(x_stride=63)),
              (I, dict(grad_y_stride=big)), (I, dict(grad_total_stride=2)), (I, dict(grad_x_stride=big)), (P, dict(x=0)), (P, dict(mean=0)),
              (P, dict(rstd=0)), (P, dict(grad_y=0)), (P, dict(workspace=0)), (S, dict(workspace_bytes=255)), (A, dict(workspace=at(9) + 16)),
              (P, dict(grad_x=at(0))), (P, dict(grad_x=at(4))), (P, dict(grad_bias=at(7))), (P, dict(grad_x=at(5), grad_x_stride=65)),
              (P, dict(grad_y=at(4, 15))), (P, dict(rstd=at(3, 1))), (A, dict(rstd=at(3) + 2))]:
    want(c, fls.fls_norm_backward, n, backward_io(**kw))
want(I, fls.fls_norm_backward, rms, backward_io())
want(I, fls.fls_norm_backward, fls.fls_norm_create(16, 64, grads=False), backward_io())
""")
    assert [x for x in got if x[0] != x[1] or x[2]] == []


def test_calls_that_are_allowed(fake):
    """In place where that is documented, without what may be left out, and without rows."""
    got = fake_cuda.run(fake, BUFFERS + """
e = fls.fls_embed_create(16, 1000, 64)
n, rms = fls.fls_norm_create(16, 64), fls.fls_norm_create(16, 64, fls.FLS_NORM_RMS)
result = []
def ok(f, h, t, launched=True):
    fake.fake_reset(0)
    result.append([code(f, h, t, stream=0), (fake.fake_launches() > 0) == launched])
ok(fls.fls_embed_lookup, e, embed_io(grad_out=0, grad_weight=0, workspace=0))
ok(fls.fls_embed_grad, e, embed_io(weight=0, out=0))
ok(fls.fls_embed_grad, e, embed_io(tokens=0, token=0, grad_out=0))
ok(fls.fls_embed_grad, e, embed_io(tokens=0, token=0, grad_out=0, accumulate=1), False)
ok(fls.fls_embed_lookup, e, embed_io(tokens=0, token=0, out=0), False)
ok(fls.fls_norm_forward, n, forward_io(total=at(0)))
ok(fls.fls_norm_forward, n, forward_io(total=at(1)))
ok(fls.fls_norm_forward, rms, forward_io(residual=0, total=0, weight=0, bias=0, mean=0, rstd=0))
ok(fls.fls_norm_forward, n, forward_io(rows=0, x=0, y=0), False)
ok(fls.fls_norm_backward, n, backward_io(grad_x=at(5)))
ok(fls.fls_norm_backward, rms, backward_io(mean=0, weight=0, grad_total=0, grad_weight=0))
ok(fls.fls_norm_backward, n, backward_io(grad_total=0, grad_x=0, grad_weight=0, grad_bias=0), False)
ok(fls.fls_norm_backward, n, backward_io(rows=0, x=0, grad_y=0, mean=0, rstd=0))
ok(fls.fls_norm_backward, n, backward_io(rows=0, x=0, grad_y=0, mean=0, rstd=0, accumulate=1), False)
""")
    assert got == [[0, True]] * len(got)


@pytest.mark.parametrize("rows,vocab,dim", [(1 << 24, 1 << 24, 16384), (1 << 24, 1, 65536), (1 << 24, 1, 1), (1, 1 << 30, 1), (1, 1 << 26, 16384),
                                            (1, 1, 65536), (131073, 128256, 2048), (131072, 128256, 2049), (0, 5, 3), (8192, 1 << 24, 8)])
@pytest.mark.parametrize("f32", [0, 1])
def test_launches_fit_the_device_at_the_largest_sizes(fake, rows, vocab, dim, f32):
    """What the create calls accept is launched: no grid beyond 65535 along y, none beyond 2^31 - 1 along x."""
    got = fake_cuda.run(fake, f"""
def place(kind, sizes, **kw):
    t, at = kind(**kw), 1 << 20
    for name, size in sizes.items():
        setattr(t, name, at)
        at += (size + 4095) // 4096 * 4096
    assert at < 1 << 44
    return t

n, V, d, size = {rows}, {vocab}, {dim}, {4 if f32 else 2}
e, norm = fls.fls_embed_create(n, V, d, True, {f32}, {f32}), fls.fls_norm_create(n, d, 1, 1e-5, {f32}, {f32}, {f32}, {f32})
ews, nws = fls.fls_embed_query(e)["workspace_bytes"], fls.fls_norm_query(norm)["workspace_bytes"]
fake.fake_reset(0)
result = [code(fls.fls_embed_lookup, e, place(fls.fls_embed_io, dict(token=8 * n, weight=2 * V * d, out=size * n * d), tokens=n, scale=1.0), stream=0)]
for accumulate in (0, 1):
    io = place(fls.fls_embed_io, dict(token=8 * n, grad_out=size * n * d, grad_weight=size * V * d, workspace=ews), tokens=n, scale=1.0,
               accumulate=accumulate, workspace_bytes=ews)
    result.append(code(fls.fls_embed_grad, e, io, stream=0))
result.append(code(fls.fls_norm_forward, norm, place(fls.fls_norm_io, dict(x=size * n * d, y=size * n * d, rstd=4 * n), rows=n), stream=0))
sizes = dict(x=size * n * d, grad_y=size * n * d, grad_x=size * n * d, rstd=4 * n, grad_weight=size * d, workspace=nws)
result.append(code(fls.fls_norm_backward, norm, place(fls.fls_norm_grad_io, sizes, rows=n, workspace_bytes=nws), stream=0))
""")
    assert got == [0] * 5


def test_reference_agrees_with_autograd_and_with_differences():
    g = torch.Generator().manual_seed(1)
    n, d = 5, 12
    for rms in (False, True):
        x = torch.randn(n, d, generator=g, dtype=torch.float64, requires_grad=True)
        w = torch.randn(d, generator=g, dtype=torch.float64, requires_grad=True)
        b = torch.randn(d, generator=g, dtype=torch.float64, requires_grad=True)
        dy = torch.randn(n, d, generator=g, dtype=torch.float64)
        y, mean, rstd = R.forward(x, w, b, 1e-5, rms)
        if not rms:
            assert torch.allclose(y, torch.nn.functional.layer_norm(x, (d,), w, b, 1e-5), atol=1e-12)
        want = torch.autograd.grad((y * dy).sum(), (x, w, b))
        got = R.backward(x.detach(), w.detach(), None if rms else mean.detach(), rstd.detach(), dy)
        assert all(torch.allclose(p, q, atol=1e-11) for p, q in zip(got, want))
        for i, j in ((0, 0), (3, 7), (4, 11)):
            step = torch.zeros(n, d, dtype=torch.float64)
            step[i, j] = 1e-6
            up, dn = ((R.forward(x.detach() + s * step, w, b, 1e-5, rms)[0] * dy).sum() for s in (1, -1))
            assert abs(float((up - dn) / 2e-6) - float(got[0][i, j])) < 1e-6
    tok = torch.tensor([3, 0, 3, -100, 7, 9, -1])
    dy = torch.randn(7, 4, generator=g)
    table = torch.zeros(9, 4, dtype=torch.float64, requires_grad=True)
    used = torch.tensor([0, 1, 2, 4])
    (table[tok[used]] * 2.5 * dy[used].double()).sum().backward()
    total, _, count = R.embed_grad(tok, dy, 9, 2.5, -100)
    assert torch.allclose(total, table.grad) and count.tolist() == [1, 0, 0, 2, 0, 0, 0, 1, 0]


def test_sources_name_no_library_product():
    for f in ("csrc/fls_embed.cu", "csrc/fls_norm.cu", "csrc/fls_elem.cuh", "embed.py", "norm.py", "workspace.py"):
        text = open(os.path.join(ROOT, "paper_2609_20359_b200", f)).read()
        assert not re.search(r"cublas|cub::|thrust|matmul|torch\.mm|einsum|index_add|layer_norm\(|triton", text, re.I), f
