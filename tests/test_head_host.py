"""CPU-side checks of the language-model head: sizes, refusals before any device is touched, and the reference itself."""
import ctypes as C
import os
import re

import pytest
import torch

from tests import head_reference as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def fls():
    from paper_2609_20359_b200 import build
    build.build()
    import paper_2609_20359_b200._binding as b
    return b


def test_struct_layouts_match_the_header(fls, tmp_path):
    import subprocess
    names = {"fls_head_desc": fls.fls_head_desc, "fls_head_layout": fls.fls_head_layout, "fls_head_io": fls.fls_head_io,
             "fls_distill_desc": fls.fls_distill_desc}
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


@pytest.mark.parametrize("kw", [dict(vocab=0), dict(dim=0), dict(dim=65537), dict(top=129), dict(max_rows=(1 << 24) + 1), dict(grad_dtype=7),
                                dict(vocab=(1 << 30) + 1), dict(max_rows=1 << 24, vocab=1 << 24), dict(piece_bytes=(1 << 40) + 1)])
def test_create_refuses(fls, kw):
    base = dict(max_rows=16, vocab=1000, dim=64)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_create(**{**base, **kw})
    assert e.value.code == fls.FLS_EINVAL and str(e.value)


def test_null_arguments(fls):
    out = C.c_void_p()
    assert fls.lib.fls_head_create(None, C.byref(out)) == fls.FLS_EINVAL
    assert fls.lib.fls_head_query(None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_head_xent(None, None, 0.0, 0.0, None) == fls.FLS_EINVAL
    assert fls.lib.fls_head_distill(None, None, None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_head_get_launch_count(None, None) == fls.FLS_EINVAL
    assert fls.lib.fls_head_get_state(None, None, None) == fls.FLS_EPTR
    assert fls.lib.fls_head_destroy(None) == fls.FLS_OK


@pytest.mark.parametrize("rows,vocab,dim,top,f32,piece", [(8192, 128256, 2048, 0, 0, 0), (1, 50257, 768, 64, 1, 0), (0, 1, 1, 0, 0, 0),
                                                          (1000, 50257, 777, 128, 1, 1 << 20), (1 << 20, 32000, 64, 0, 0, 0)])
def test_workspace_and_pieces(fls, rows, vocab, dim, top, f32, piece):
    h = fls.fls_head_create(rows, vocab, dim, top, True, f32, False, piece)
    q = fls.fls_head_query(h)
    cap, planes = max(256, -(-rows // 256) * 256), 2 if f32 else 1
    # the kept columns at the end (4 bytes each, whole tiles of 256) and the pieces before them cover the vocabulary once
    formed, most = vocab - q["kept_cols"], max(piece or 1 << 30, 2 * planes * cap * 512)
    assert 0 <= q["kept_cols"] <= vocab and (formed == 0 or formed % 256 == 0 or q["kept_cols"] == 0)
    assert q["piece_cols"] % 256 == 0 and q["piece_cols"] * q["pieces"] >= formed and (formed == 0) == (q["pieces"] == 0)
    assert q["pieces"] == 0 or formed > q["piece_cols"] * (q["pieces"] - 1)
    assert 4 * cap * (-(-q["kept_cols"] // 256) * 256) <= most
    g = max(2 * planes * cap * q["piece_cols"], 4 * cap * q["kept_cols"])
    assert g <= most
    assert q["workspace_bytes"] >= g + 2 * cap * dim
    less = fls.fls_head_create(rows, vocab, dim, top, False, f32, False, piece)
    assert fls.fls_head_query(less)["workspace_bytes"] < q["workspace_bytes"]
    fls.fls_head_destroy(less)
    fls.fls_head_destroy(h)


def _io(fls, **kw):
    io = fls.fls_head_io()
    io.rows, io.ignore_label = 4, -100
    for k, v in kw.items():
        setattr(io, k, v)
    return io


@pytest.mark.parametrize("kw,code", [(dict(rows=17), "FLS_EINVAL"), (dict(reserved=1), "FLS_EINVAL"), (dict(accumulate=2), "FLS_EINVAL"),
                                     (dict(hidden_stride=63), "FLS_EINVAL"), (dict(weight_stride=1 << 40), "FLS_EINVAL"),
                                     (dict(weight=8), "FLS_EALIGN"), (dict(weight=16, weight_stride=65), "FLS_EALIGN"), (dict(), "FLS_EPTR"),
                                     (dict(hidden=1), "FLS_EALIGN"), (dict(workspace=256, workspace_bytes=100), "FLS_ESIZE")])
def test_call_refuses_before_it_needs_a_device(fls, kw, code):
    h = fls.fls_head_create(16, 1000, 64)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_xent(h, _io(fls, **kw), stream=0)
    assert e.value.code == getattr(fls, code)
    fls.fls_head_destroy(h)


@pytest.mark.parametrize("eps,zeta", [(-0.1, 0.0), (1.0, 0.0), (float("nan"), 0.0), (0.0, -1.0), (0.0, float("inf"))])
def test_xent_refuses_its_options(fls, eps, zeta):
    h = fls.fls_head_create(16, 1000, 64)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_xent(h, _io(fls), eps, zeta, stream=0)
    assert e.value.code == fls.FLS_EINVAL
    fls.fls_head_destroy(h)


@pytest.mark.parametrize("kw,top", [(dict(temperature=0.0), 4), (dict(temperature=float("nan")), 4), (dict(temperature=float("inf")), 4),
                                    (dict(tail=2), 4), (dict(distill_weight=-1.0), 4), (dict(label_weight=float("nan")), 4),
                                    (dict(reserved=1), 4), (dict(), 0)])
def test_distill_refuses_its_options(fls, kw, top):
    h = fls.fls_head_create(16, 1000, 64, top)
    t = fls.fls_distill_desc(temperature=1.0, distill_weight=1.0)
    for k, v in kw.items():
        setattr(t, k, v)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_distill(h, _io(fls), t, stream=0)
    assert e.value.code == fls.FLS_EINVAL
    fls.fls_head_destroy(h)


def test_gradients_need_a_head_made_for_them(fls):
    h = fls.fls_head_create(16, 1000, 64, grads=False)
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_xent(h, _io(fls, grad_hidden=256), stream=0)
    assert e.value.code == fls.FLS_EINVAL
    fls.fls_head_destroy(h)


def test_reference_agrees_with_torch_and_with_differences():
    """The 64-bit forms the kernels are compared with: torch's own losses, and central differences of the loss."""
    g = torch.Generator().manual_seed(3)
    n, V, k = 6, 40, 5
    z = torch.randn(n, V, generator=g, dtype=torch.float64)
    y = torch.randint(0, V, (n,), generator=g)
    y[1] = -100
    live = y >= 0
    loss, lse = R.xent_rows(z, y, live, 0.1, 0.0)
    want = torch.nn.functional.cross_entropy(z, y, ignore_index=-100, label_smoothing=0.1, reduction="none")
    assert torch.allclose(loss, want, atol=1e-12)
    idx = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(n)]).to(torch.int32)
    t = torch.randn(n, k, generator=g)
    T = 2.0
    loss, _, _ = R.distill_rows(z, idx, t, y, T, 1.0, 0.0, None, -100)
    q = torch.full((n, V), -torch.inf, dtype=torch.float64).scatter(1, idx.long(), t.double()).div(T).softmax(1)
    want = torch.nn.functional.kl_div(torch.log_softmax(z / T, 1), q, reduction="none").sum(1) * T * T
    assert torch.allclose(loss, want, atol=1e-12)
    tl = torch.logsumexp(t.double() / T, 1) + 0.3
    zz = z.clone().requires_grad_(True)
    R.distill_rows(zz, idx, t, y, T, 0.7, 0.3, tl, -100)[0].sum().backward()
    for i, j in ((0, int(idx[0, 0])), (0, int(y[0])), (1, 7), (5, 39), (3, int(idx[3, 4]))):
        e = torch.zeros_like(z)
        e[i, j] = 1e-5
        up, dn = (R.distill_rows(z + s * e, idx, t, y, T, 0.7, 0.3, tl, -100)[0].sum() for s in (1, -1))
        assert abs(float((up - dn) / 2e-5) - float(zz.grad[i, j])) < 1e-8


def test_head_sources_name_no_library_product():
    """The head's own kernels do its products: no cuBLAS, no torch matrix product in the binding."""
    for f in ("csrc/fls_head_kernels.cu", "csrc/fls_head_api.cu", "head.py"):
        text = open(os.path.join(ROOT, "paper_2609_20359_b200", f)).read()
        assert not re.search(r"cublas|matmul|torch\.mm|einsum|\.softmax|triton", text, re.I), f
