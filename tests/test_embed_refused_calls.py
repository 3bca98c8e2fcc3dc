"""A call that was refused has no say in the next one."""
import pytest
import torch

from tests.test_embed_norm_threads import host  # noqa: F401

FAR = 1 << 31                                               # elements between rows that the library refuses


@pytest.fixture
def embedding(host):
    from paper_2609_20359_b200 import embed
    host.setattr(embed, "matrix", lambda t, name, rows, cols, dtype: (t.data_ptr(), t.stride(0)))
    return embed.Embedding(4, 10, 8)


def rows(n, stride=8):
    return torch.empty_strided((n, 8), (stride, 1), dtype=torch.bfloat16)


NONE = torch.empty(0, dtype=torch.int64)


def code(f, *args, **kw):
    from paper_2609_20359_b200 import _binding as fls
    try:
        f(*args, **kw)
    except fls.FlsError as e:
        return e.code
    return fls.FLS_OK


@pytest.mark.parametrize("which", ["grad_out", "grad_weight"])
def test_lookup_after_a_refused_gradient(embedding, which):
    from paper_2609_20359_b200 import _binding as fls
    table = rows(10)
    dy, gw = rows(0, FAR if which == "grad_out" else 8), rows(0, FAR if which == "grad_weight" else 8)
    assert code(embedding.grad, NONE, dy, gw) == fls.FLS_EINVAL
    assert code(embedding.lookup, NONE, table) == fls.FLS_OK


@pytest.mark.parametrize("which", ["weight", "out"])
def test_gradient_after_a_refused_lookup(embedding, which):
    from paper_2609_20359_b200 import _binding as fls
    table, out = rows(0, FAR if which == "weight" else 8), rows(0, FAR if which == "out" else 8)
    assert code(embedding.lookup, NONE, table, out=out) == fls.FLS_EINVAL
    # the strides are accepted; that the buffers are not on a device is seen after them
    assert code(embedding.grad, NONE, rows(0), rows(10)) in (fls.FLS_EPTR, fls.FLS_ECUDA)
