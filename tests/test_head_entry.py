"""What the entry points of the head and of the top logits refuse and launch, seen on a CUDA runtime that only writes it down."""
import pytest

from tests import fake_cuda


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    return fake_cuda.build(tmp_path_factory.mktemp("fake"))


def test_buffers_of_another_device_are_refused(fake):
    """Each buffer in turn on a device that is not the current one, and on the host; then all where they belong."""
    got = fake_cuda.run(fake, """
def top(**kw):
    at = lambda i, d=1: (d << 44) + (i + 1 << 24)
    p = dict(logits=at(0), value=at(1), index=at(2), lse=at(3), **{})
    p.update({k: at(["logits", "value", "index", "lse"].index(k), d) for k, d in kw.items()})
    return fls.fls_top_logits(p["logits"], fls.FLS_GRAD_BF16, 3, 1000, 0, 5, 1.0, p["value"], p["index"], p["lse"], stream=0)

result = {"top": [], "head": []}
fake.fake_reset(1)
for owner in (0, 2, 15):
    result["top"] += [[code(top, **{k: owner}), fake.fake_launches()] for k in ("logits", "value", "index", "lse")]
result["top ok"] = [code(top), fake.fake_launches()]
head = fls.fls_head_create(64, 1000, 64)
lay = fls.fls_head_query(head)
fake.fake_reset(1)
for owner in (0, 15):
    for name in ("hidden", "weight", "labels", "loss", "lse", "grad_hidden", "grad_weight", "workspace"):
        io = buffers(64, 1000, 64, lay, device=1)
        setattr(io, name, getattr(io, name) % (1 << 44) + (owner << 44))
        result["head"].append([code(fls.fls_head_xent, head, io, stream=0), fake.fake_launches()])
result["head ok"] = [code(fls.fls_head_xent, head, buffers(64, 1000, 64, lay, device=1), stream=0), fake.fake_launches() > 0]
result["EPTR"] = fls.FLS_EPTR
""")
    assert got["top"] == [[got["EPTR"], 0]] * 12 and got["top ok"] == [0, 1]
    assert got["head"] == [[got["EPTR"], 0]] * 16 and got["head ok"] == [0, True]


def test_star_import_has_every_entry_point():
    """`from ..._binding import *` gives all that the library exports and the structures its calls take."""
    from paper_2609_20359_b200 import _binding as b
    names = {}
    exec("from paper_2609_20359_b200._binding import *", names)
    assert [n for n in b.EXPORTS if n not in names] == []
    assert all(n in names for n in ("fls_head_desc", "fls_head_io", "fls_distill_desc", "FLS_TAIL_CLASS", "FLS_HEAD_MAX_TOP"))


def test_a_call_without_rows_counts_none(fake):
    """The word behind rows_taking_part is cleared or rewritten by every call that has no rows."""
    got = fake_cuda.run(fake, """
head = fls.fls_head_create(64, 1000, 64)
lay = fls.fls_head_query(head)
result = []
for grads, accumulate in ((False, 0), (True, 0), (True, 1)):
    fake.fake_reset(0)
    io = buffers(0, 1000, 64, lay, grads)
    io.accumulate = accumulate
    rc = code(fls.fls_head_xent, head, io, stream=0)
    count = fls.fls_head_get_state(io.workspace)[1]
    result.append([rc, fake.fake_launches() > 0, clears() == [[count, 4]]])
""")
    assert got == [[0, False, True], [0, True, False], [0, False, True]]


@pytest.mark.gpu
def test_rows_taking_part_after_a_call_without_rows():
    import torch
    from paper_2609_20359_b200.head import Head
    dev, V, d = "cuda:0", 300, 64
    h = torch.randn(5, d, device=dev).bfloat16()
    w = torch.randn(V, d, device=dev).bfloat16()
    y = torch.arange(5, device=dev)
    gw = torch.zeros_like(w)
    head = Head(8, V, d)
    for kw in (dict(), dict(grad_weight=gw), dict(grad_weight=gw, accumulate=True)):
        head.xent(h, w, y)
        assert int(head.rows_taking_part()) == 5
        head.xent_step(h[:0], w, y[:0], **kw)
        assert int(head.rows_taking_part()) == 0


@pytest.mark.parametrize("rows,vocab,dim", [(300, 1 << 27, 8), (1 << 24, 1 << 23, 8), (256, 1 << 30, 16), (8192, 128256, 2048), (1, 1, 65536)])
def test_groups_of_row_tiles_fit_32_bits(fake, rows, vocab, dim):
    """The statistics' schedule counts tiles of a group in 32 bits: row tiles of the group times column tiles."""
    got = fake_cuda.run(fake, f"""
head = fls.fls_head_create({rows}, {vocab}, {dim}, grads=False)
io = buffers({rows}, {vocab}, {dim}, fls.fls_head_query(head), False)
fake.fake_reset(0)
result = [code(fls.fls_head_xent, head, io, stream=0), fake.fake_group_m()]
""")
    assert got[0] == 0
    assert 1 <= got[1] and got[1] * -(-vocab // 256) < 1 << 32
    assert got[1] == max(1, min(-(-rows // 256), (32 << 20) // (256 * dim * 2)))


@pytest.mark.parametrize("rows,vocab,dim,top,f32,any_weight,piece", [
    (1 << 24, 1000, 896, 0, 0, 0, 0), (1 << 24, 1000, 896, 128, 1, 0, 0), (8388480, 300, 1024, 0, 0, 0, 0),
    (8388481, 300, 1024, 0, 0, 0, 0), (1, 1 << 30, 8, 0, 0, 1, 1 << 36), (256, 1 << 28, 1024, 0, 0, 0, 1 << 40),
    (1, 2, 65536, 1, 1, 1, 0)])
def test_launches_fit_the_device_at_the_largest_sizes(fake, rows, vocab, dim, top, f32, any_weight, piece):
    """What fls_head_create accepts is launched: no grid beyond 65535 along y, none beyond 2^31 - 1 along x."""
    got = fake_cuda.run(fake, f"""
head = fls.fls_head_create({rows}, {vocab}, {dim}, {top}, True, {f32}, bool({any_weight}), {piece})
io = buffers({rows}, {vocab}, {dim}, fls.fls_head_query(head), True, {f32})
fake.fake_reset(0)
result = [code(fls.fls_head_xent, head, io, stream=0)]
if {top}:
    fake.fake_reset(0)
    t = fls.fls_distill_desc(1 << 43, (1 << 43) + (1 << 41), (1 << 43) + (1 << 42), fls.FLS_TAIL_CLASS, 0, 2.0, 0.5, 0.5)
    result.append(code(fls.fls_head_distill, head, io, t, stream=0))
result.append(fake.fake_launches())
""")
    assert not any(got[:-1]) and got[-1] >= 5
