"""GPU tests of the language-model head against plain 64-bit forms, at the sizes and masks where it can go wrong."""
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


def make(n, V, d, seed=0, scale=2.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, d, generator=g, device=DEV) * (scale / math.sqrt(d))).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV)
    return h, w, y, g


def buffers(n, V, d, f32=False):
    """Outputs filled with NaN: what is not written shows."""
    gh = torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV)
    gw = torch.full((V, d), math.nan, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    return gh, gw


def xent_case(n, V, d, f32=False, eps=0.0, zeta=0.0, ignored=(), piece=0, row_weight=None, seed=0, head=None):
    from paper_2609_20359_b200.head import Head
    h, w, y, _ = make(n, V, d, seed)
    for i in ignored:
        y[i] = IGN
    gh, gw = buffers(n, V, d, f32)
    head = head or Head(n, V, d, grad_dtype="f32" if f32 else "bf16", piece_bytes=piece)
    loss, lse = head.xent_step(h, w, y, gh, gw, row_weight=row_weight, label_smoothing=eps, z_loss=zeta)
    live = y != IGN
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, eps, zeta), live), row_weight)
    R.check_rows(ref, loss, lse, 1 + 2 * zeta * float(ref["lse"].abs().max() if n else 0))
    R.check_grads(ref, gh, gw)
    assert head.status() == 0 and int(head.rows_taking_part()) == int(live.sum())
    return head


# one row to several row tiles; vocabularies around the 256-column tile and the 64-deep stage; depths around 64 and off 8
@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 257])
@pytest.mark.parametrize("V,d", [(1, 8), (7, 64), (256, 64), (257, 72), (1000, 136)])
def test_xent_sizes(n, V, d):
    xent_case(n, V, d)


@pytest.mark.parametrize("d", [1, 3, 63, 65, 250, 257])
@pytest.mark.parametrize("f32", [False, True])
def test_xent_depths_off_the_grid(d, f32):
    xent_case(33, 515, d, f32=f32)


@pytest.mark.parametrize("eps,zeta", [(0.1, 0.0), (0.0, 1e-2), (0.2, 1e-3)])
@pytest.mark.parametrize("f32", [False, True])
def test_xent_smoothing_and_z_loss(eps, zeta, f32):
    xent_case(200, 3001, 128, f32=f32, eps=eps, zeta=zeta, ignored=(0, 199))


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n,V,d,piece", [(300, 5003, 96, 1), (700, 2500, 320, 1 << 20), (64, 40000, 64, 1 << 22)])
def test_xent_in_several_pieces(n, V, d, piece, f32):
    head = xent_case(n, V, d, f32=f32, piece=piece)
    assert head.layout["pieces"] > 1


@pytest.mark.parametrize("n,V,d", [(2048, 20000, 512), (1025, 50257, 768), (3, 128256, 2048)])
def test_xent_larger(n, V, d):
    xent_case(n, V, d, ignored=range(0, n, 3) if n > 3 else ())


# wide enough for kept logits: all of them, a part of them, none; one and two terms of dL/dz
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("n,V,d,piece", [(1, 300, 896, 0), (130, 777, 1000, 0), (300, 3000, 904, 1 << 22), (300, 3000, 904, 1)])
def test_xent_kept_columns(n, V, d, piece, f32):
    head = xent_case(n, V, d, f32=f32, piece=piece, eps=0.1, zeta=1e-3, ignored=(0,) if n > 1 else ())
    assert (head.layout["kept_cols"] == V) == (piece == 0) and (head.layout["pieces"] == 0) == (piece == 0)


def test_kept_and_formed_logits_give_the_same_bits():
    from paper_2609_20359_b200.head import Head
    n, V, d, k = 200, 2600, 1024, 9
    h, w, y, g = make(n, V, d)
    idx, t = teacher(n, V, k, g)
    outs = []
    for piece in (0, 1 << 20):
        gh, gw = buffers(n, V, d, True)
        head = Head(n, V, d, top=k, grad_dtype="f32", piece_bytes=piece)
        outs.append((head.layout["kept_cols"], *head.distill_step(h, w, idx, t, gh, gw, labels=y, temperature=2.0, label_weight=0.4), gw))
    assert outs[0][0] == V > outs[1][0]
    assert all(torch.equal(a, b) for a, b in zip(outs[0][1:], outs[1][1:]))


def test_smaller_calls_of_one_head():
    from paper_2609_20359_b200.head import Head
    head = Head(600, 1300, 128, piece_bytes=1 << 20)
    for n in (600, 1, 300, 5, 599):
        xent_case(n, 1300, 128, head=head, seed=n)


def test_row_weights():
    rw = torch.rand(90, device=DEV) * 3 - 1
    rw[5] = 0.0
    xent_case(90, 700, 64, row_weight=rw, ignored=(7,))


@pytest.mark.parametrize("which", ["hidden", "weight"])
def test_one_gradient_alone(which):
    from paper_2609_20359_b200.head import Head
    n, V, d = 150, 900, 192
    h, w, y, _ = make(n, V, d)
    gh, gw = buffers(n, V, d)
    head = Head(n, V, d)
    both = (gh.clone(), gw.clone())
    head.xent_step(h, w, y, *both)
    if which == "hidden":
        head.xent_step(h, w, y, grad_hidden=gh)
        assert torch.equal(gh, both[0])
    else:
        head.xent_step(h, w, y, grad_weight=gw)
        assert torch.equal(gw, both[1])


def test_same_inputs_same_bits():
    from paper_2609_20359_b200.head import Head
    n, V, d = 400, 6000, 256
    h, w, y, _ = make(n, V, d)
    head = Head(n, V, d, piece_bytes=1 << 20)
    first = None
    for _ in range(4):
        gh, gw = buffers(n, V, d)
        out = (*head.xent_step(h, w, y, gh, gw), gh, gw)
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))


@pytest.mark.parametrize("f32", [False, True])
def test_accumulate(f32):
    from paper_2609_20359_b200.head import Head
    n, V, d = 70, 600, 100
    h, w, y, _ = make(n, V, d)
    live = torch.ones(n, dtype=torch.bool, device=DEV)
    head = Head(n, V, d, grad_dtype="f32" if f32 else "bf16")
    gw = torch.randn(V, d, device=DEV).to(torch.float32 if f32 else torch.bfloat16)
    before = gw.clone()
    head.xent_step(h, w, y, grad_weight=gw, accumulate=True)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    ref["grad_weight"] = ref["grad_weight"] + before.double()
    R.check_grads(ref, grad_weight=gw)
    none = torch.full_like(y, IGN)
    kept = gw.clone()
    head.xent_step(h, w, none, grad_weight=gw, accumulate=True)
    assert torch.equal(gw, kept)


@pytest.mark.parametrize("off,extra", [(0, 0), (0, 8), (8, 24), (1, 3), (3, 0)])
@pytest.mark.parametrize("d", [64, 100])
def test_strides_and_alignment(off, extra, d):
    """Views into wider, offset buffers; what lies between the rows stays as it was."""
    from paper_2609_20359_b200.head import Head
    n, V = 130, 530
    h0, w0, y, _ = make(n, V, d)

    def view(rows, dtype, fill):
        buf = torch.full((off + rows * (d + extra) + 8,), fill, dtype=dtype, device=DEV)
        return buf, buf[off: off + rows * (d + extra)].view(rows, d + extra)[:, :d]

    (_, h), (_, w) = view(n, torch.bfloat16, 7.0), view(V, torch.bfloat16, 7.0)
    h.copy_(h0)
    w.copy_(w0)
    (bh, gh), (bw, gw) = view(n, torch.bfloat16, 5.0), view(V, torch.bfloat16, 5.0)
    head = Head(n, V, d, any_weight=True)
    loss, lse = head.xent_step(h, w, y, gh, gw)
    live = torch.ones(n, dtype=torch.bool, device=DEV)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    R.check_rows(ref, loss, lse)
    R.check_grads(ref, gh, gw)
    for b, v in ((bh, gh), (bw, gw)):
        v.fill_(5.0)
        assert bool((b == 5.0).all())


def test_rows_without_a_label_may_hold_anything():
    """NaN and infinity in ignored rows reach nothing; a call whose every row is ignored writes zeros."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 260, 700, 128
    h, w, y, _ = make(n, V, d)
    y[::2] = IGN
    h[0], h[2], h[258] = math.nan, math.inf, -math.inf
    head = Head(n, V, d)
    gh, gw = buffers(n, V, d)
    loss, lse = head.xent_step(h, w, y, gh, gw)
    live = y != IGN
    clean = torch.where(live[:, None], h, 0.0)
    ref = R.with_gradients(clean, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    R.check_rows(ref, loss, lse)
    R.check_grads(ref, gh, gw)
    assert bool((gh[::2] == 0).all()) and bool((loss[::2] == 0).all())
    y[:] = IGN
    gh, gw = buffers(n, V, d)
    loss, lse = head.xent_step(h, w, y, gh, gw)
    assert not any(bool(t.any()) for t in (loss, lse, gh, gw)) and int(head.rows_taking_part()) == 0


def test_labels_outside_the_vocabulary():
    from paper_2609_20359_b200.head import Head
    n, V, d = 20, 300, 64
    h, w, y, _ = make(n, V, d)
    y[3], y[4], y[5] = V, -1, IGN
    head = Head(n, V, d)
    gh, gw = buffers(n, V, d)
    loss, _ = head.xent_step(h, w, y, gh, gw)
    assert torch.isnan(loss).nonzero()[:, 0].tolist() == [3, 4] and float(loss[5]) == 0.0
    live = (y >= 0) & (y < V)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    R.check_grads(ref, gh, gw)


def test_nan_in_one_row_stays_in_that_row():
    from paper_2609_20359_b200.head import Head
    n, V, d = 40, 600, 64
    h, w, y, _ = make(n, V, d)
    head = Head(n, V, d)
    gh0, _ = buffers(n, V, d)
    loss0, _ = head.xent_step(h, w, y, gh0)
    h[11, 5] = math.nan
    gh, _ = buffers(n, V, d)
    loss, lse = head.xent_step(h, w, y, gh)
    others = torch.arange(n, device=DEV) != 11
    assert bool(torch.isnan(loss[11])) and bool(torch.isnan(lse[11])) and bool(torch.isnan(gh[11]).all())
    assert torch.equal(loss[others], loss0[others]) and torch.equal(gh[others], gh0[others])


def test_confident_rows_keep_their_digits():
    """p_label close to 1: the loss is log1p of the rest, not a difference of two large numbers."""
    from paper_2609_20359_b200.head import Head
    V, d = 400, 64
    w = torch.zeros(V, d, device=DEV, dtype=torch.bfloat16)
    w[0, 0] = 1.0
    h = torch.zeros(5, d, device=DEV, dtype=torch.bfloat16)
    h[:, 0] = torch.tensor([20.0, 30.0, 60.0, 90.0, -90.0], device=DEV)
    y = torch.zeros(5, dtype=torch.int64, device=DEV)
    gh, _ = buffers(5, V, d)
    loss, _ = Head(5, V, d).xent_step(h, w, y, gh, row_weight=torch.ones(5, device=DEV))
    z = h[:, 0].double()
    want = torch.log1p((V - 1) * torch.exp(-z))
    assert bool(((loss.double() - want).abs() <= 1e-5 * want).all())
    # dL/dh = sum_v p_v w_v - w_0: only column 0 carries weight
    grad = -((V - 1) * torch.exp(-z)) / (1 + (V - 1) * torch.exp(-z))
    assert bool(((gh[:, 0].double() - grad).abs() <= 2.0 ** -7 * grad.abs()).all())


def test_large_logits():
    from paper_2609_20359_b200.head import Head
    n, V, d = 30, 900, 64
    h, w, y, _ = make(n, V, d, scale=200.0)
    gh, gw = buffers(n, V, d)
    loss, lse = Head(n, V, d).xent_step(h, w, y, gh, gw)
    live = torch.ones(n, dtype=torch.bool, device=DEV)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    R.check_rows(ref, loss, lse)
    assert bool(torch.isfinite(gh).all()) and bool(torch.isfinite(gw).all())


def test_gradient_against_differences_of_the_loss():
    """Central differences of the kernel's own loss; steps that bf16 holds exactly."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 12, 500, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    h = (torch.randint(-8, 9, (n, d), generator=g, device=DEV) / 8).bfloat16()
    _, w, y, _ = make(n, V, d, 5)
    head = Head(n, V, d, grad_dtype="f32")
    gh, gw = buffers(n, V, d, True)
    head.xent_step(h, w, y, gh, gw, label_smoothing=0.1, z_loss=1e-3, row_weight=torch.ones(n, device=DEV))
    e = 2.0 ** -5
    for i in (0, 17, 63):
        up, dn = h.clone(), h.clone()
        up[:, i] += e
        dn[:, i] -= e
        lu, ld = (head.xent(x, w, y, label_smoothing=0.1, z_loss=1e-3)[0].double() for x in (up, dn))
        diff = (lu - ld) / (2 * e)
        # third derivative of the loss along one coordinate: below 2 * max|w|^3 for softmax losses; then bf16 of the gradient
        # and of dL/dz, and fp32 losses of size 10
        lim = e * e / 6 * 4 * float(w[:, i].abs().max()) ** 3 + 2.0 ** -7 * (1 + float(w[:, i].abs().max())) * 0.25 + 2e-6 / e
        assert bool(((diff - gh[:, i].double()).abs() <= lim).all())


def test_two_streams():
    """Two heads on two streams, their inputs written on those streams."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 300, 4000, 256
    jobs = []
    for k in range(2):
        s = torch.cuda.Stream()
        head = Head(n, V, d)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            h, w, y, _ = make(n, V, d, seed=k)
            gh, gw = buffers(n, V, d)
        loss, lse = head.xent_step(h, w, y, gh, gw, stream=s)
        jobs.append((h, w, y, gh, gw, loss, lse))
    torch.cuda.synchronize()
    for h, w, y, gh, gw, loss, lse in jobs:
        live = torch.ones(n, dtype=torch.bool, device=DEV)
        ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
        R.check_rows(ref, loss, lse)
        R.check_grads(ref, gh, gw)


def test_graph_capture():
    from paper_2609_20359_b200.head import Head
    n, V, d = 100, 2000, 128
    h, w, y, _ = make(n, V, d)
    gh, gw = buffers(n, V, d)
    head = Head(n, V, d)
    want = [t.clone() for t in (*head.xent_step(h, w, y, gh, gw), gh, gw)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, lse = head.xent_step(h, w, y, gh, gw)
    gh.zero_()
    gw.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, gh, gw)))


def test_writes_into_a_gradient_buffer_of_a_session():
    """The head's unit of a plan's flat gradient buffer is a valid grad_weight; nothing else of the buffer changes."""
    from paper_2609_20359_b200.head import Head
    from paper_2609_20359_b200.session import Session
    n, V, d = 60, 501, 64
    s = Session(V * d + 1000, [V * d, 1000], groups=2, shard_dim=2)
    h, w, y, _ = make(n, V, d)
    off = s.layout["unit_offset"][0]
    for row in s.grads:
        for b in row:
            b.fill_(3.0)
    gw = s.grads[1][0][off: off + V * d].view(V, d)
    head = Head(n, V, d)
    head.xent_step(h, w, y, grad_weight=gw)
    _, want = buffers(n, V, d)
    head.xent_step(h, w, y, grad_weight=want)
    assert torch.equal(gw, want)
    assert bool((s.grads[1][0][off + V * d:] == 3.0).all()) and bool((s.grads[0][0] == 3.0).all())


# ------------------------------------------------------------------------------------------------ distillation
def teacher(n, V, k, g, ragged=True):
    idx = torch.stack([torch.randperm(V, generator=g, device=DEV)[:k] for _ in range(n)]).to(torch.int32)
    t = 3 * torch.randn(n, k, generator=g, device=DEV)
    if ragged and n > 3 and k > 1:
        idx[1, k // 2:] = -1
        t[2, 0] = -math.inf
        idx[3, k - 1] = V + 5
    return idx, t


def distill_case(n, V, d, k, T=1.0, tail=False, wl=0.0, wd=1.0, f32=False, piece=0, ignored=(), empty=(), seed=0):
    from paper_2609_20359_b200.head import Head
    h, w, y, g = make(n, V, d, seed)
    idx, t = teacher(n, V, k, g)
    for i in ignored:
        y[i] = IGN
    for i in empty:
        idx[i] = -1
    if n > 5 and wl:
        y[5] = idx[5, 0]                       # a label that is in the teacher's list
    tl = None
    if tail:
        ok = (idx >= 0) & (idx < V)
        tl = torch.logsumexp((t / T).masked_fill(~ok, -math.inf), 1) + 0.05 + torch.rand(n, generator=g, device=DEV)
        tl = torch.where(torch.isfinite(tl), tl, 0.0)
    gh, gw = buffers(n, V, d, f32)
    head = Head(n, V, d, top=k, grad_dtype="f32" if f32 else "bf16", piece_bytes=piece)
    kw = dict(labels=y, teacher_lse=tl, temperature=T, distill_weight=wd, label_weight=wl)
    loss, lse = head.distill_step(h, w, idx, t, gh, gw, **kw)
    ref = R.with_gradients(h, w, lambda z: R.distill_rows(z, idx, t, y, T, wd, wl, tl, IGN))
    # q' = 1 - sum q is known to 2^-53 only, q itself to 2^-24 of its input: the tail's gradient and loss inherit that
    R.check_rows(ref, loss, lse, wd * T * T + wl + (8 * T * T if tail else 0), T)
    R.check_grads(ref, gh, gw)
    alone = head.distill(h, w, idx, t, **kw)
    assert torch.equal(alone[0], loss) and torch.equal(alone[1], lse)
    assert int(head.rows_taking_part()) == int(ref["live"].sum()) and head.status() == 0


@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 128])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,wl", [(1.0, 0.0), (2.0, 0.0), (1.0, 0.5), (2.5, 0.5)])
def test_distill_lists(k, tail, T, wl):
    distill_case(40, 700, 64, k, T, tail, wl, 0.8, ignored=(4, 6), empty=(6, 7))


@pytest.mark.parametrize("n,V,d,k", [(1, 300, 64, 8), (129, 257, 72, 16), (300, 5000, 256, 64), (20, 128, 64, 128)])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_sizes(n, V, d, k, tail):
    if tail and k == V:
        pytest.skip("no column outside the list: its class has probability zero")
    distill_case(n, V, d, k, 2.0, tail, 0.5)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,wl", [(1.0, 0.0), (3.0, 0.5)])
def test_distill_kept_columns(f32, tail, T, wl):
    distill_case(140, 1500, 912, 40, T, tail, wl, f32=f32, ignored=(4, 6), empty=(6, 7))
    distill_case(140, 1500, 912, 40, T, tail, wl, f32=f32, piece=1 << 20)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_in_several_pieces(f32, tail):
    distill_case(257, 3000, 128, 20, 1.5, tail, 0.3, f32=f32, piece=1)


def test_distill_rows_without_a_teacher_may_hold_anything():
    from paper_2609_20359_b200.head import Head
    n, V, d, k = 50, 400, 64, 6
    h, w, y, g = make(n, V, d)
    idx, t = teacher(n, V, k, g, ragged=False)
    idx[10] = -1
    t[11] = -math.inf
    h[10], h[11] = math.nan, math.inf
    gh, gw = buffers(n, V, d)
    loss, lse = Head(n, V, d, top=k).distill_step(h, w, idx, t, gh, gw)
    clean = h.clone()
    clean[10:12] = 0
    ref = R.with_gradients(clean, w, lambda z: R.distill_rows(z, idx, t, y, 1.0, 1.0, 0.0, None, IGN))
    R.check_rows(ref, loss, lse)
    R.check_grads(ref, gh, gw)
    assert not bool(gh[10:12].any()) and not bool(loss[10:12].any())


def test_teacher_entries_at_the_lowest_value():
    """Entries masked with the type's lowest value have probability zero, and a list of nothing else is uniform."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 9, 300, 64
    h, w, y, g = make(n, V, d)
    idx, t = teacher(n, V, 6, g, ragged=False)
    t[:, 2] = torch.finfo(torch.float32).min
    t[4] = torch.finfo(torch.float32).min
    gh, gw = buffers(n, V, d)
    loss, lse = Head(n, V, d, top=6).distill_step(h, w, idx, t, gh, gw, temperature=0.5)
    ref = R.with_gradients(h, w, lambda z: R.distill_rows(z, idx, t, y, 0.5, 1.0, 0.0, None, IGN))
    R.check_rows(ref, loss, lse, 1.0, 0.5)
    R.check_grads(ref, gh, gw)


@pytest.mark.parametrize("n,V,d", [(1, 700, 64), (300, 3000, 1024)])
def test_the_loss_alone_is_that_of_the_step(n, V, d):
    from paper_2609_20359_b200.head import Head
    h, w, y, _ = make(n, V, d)
    gh, gw = buffers(n, V, d)
    full, lean = Head(n, V, d), Head(n, V, d, grads=False)
    step = full.xent_step(h, w, y, gh, gw, label_smoothing=0.1)
    for head in (full, lean):
        assert all(torch.equal(a, b) for a, b in zip(step, head.xent(h, w, y, label_smoothing=0.1)))


def test_repeated_teacher_entries_add_up():
    """Two entries on one column count as two entries: in the gradient their probabilities add."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 9, 300, 64
    h, w, y, g = make(n, V, d)
    idx, t = teacher(n, V, 4, g, ragged=False)
    idx[:, 3] = idx[:, 1]
    gh, gw = buffers(n, V, d)
    loss, lse = Head(n, V, d, top=4).distill_step(h, w, idx, t, gh, gw)
    ref = R.with_gradients(h, w, lambda z: R.distill_rows(z, idx, t, y, 1.0, 1.0, 0.0, None, IGN))
    R.check_rows(ref, loss, lse)
    R.check_grads(ref, gh, gw)


# ------------------------------------------------------------------------------------------------ refusals
def test_refusals_on_the_device():
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.head import Head
    n, V, d = 8, 100, 64
    h, w, y, _ = make(n, V, d)
    head = Head(n, V, d)
    gh, gw = buffers(n, V, d)
    with pytest.raises(fls.FlsError) as e:
        head.xent_step(h, w, y, grad_hidden=h)
    assert e.value.code == fls.FLS_EPTR and "overlaps" in str(e.value)
    with pytest.raises(fls.FlsError) as e:
        head.xent_step(h, w, y, grad_hidden=w[:n])
    assert e.value.code == fls.FLS_EPTR
    odd = torch.empty(V * d + 1, dtype=torch.bfloat16, device=DEV)[1:].view(V, d)
    with pytest.raises(fls.FlsError) as e:
        head.xent(h, odd, y)
    assert e.value.code == fls.FLS_EALIGN
    io, _ = head._io(h, w, y, IGN, None, None, None, False, None)
    host = torch.empty(n, dtype=torch.float32)
    io.loss = host.data_ptr()
    with pytest.raises(fls.FlsError) as e:
        fls.fls_head_xent(head.handle, io)
    assert e.value.code == fls.FLS_EPTR and "device memory" in str(e.value)
    for bad in (dict(hidden=h.float()), dict(hidden=h[:, :32]), dict(labels=y.int()), dict(labels=y[:4]), dict(weight=w.t().contiguous().t()),
                dict(hidden=h.cpu())):
        with pytest.raises(ValueError):
            head.xent(**{"hidden": h, "weight": w, "labels": y, **bad})
    with pytest.raises(ValueError):
        head.xent_step(h, w, y, grad_weight=gw.float())
    with pytest.raises(fls.FlsError):
        head.distill(h, w, torch.empty(n, 0, dtype=torch.int32, device=DEV), torch.empty(n, 0, device=DEV))


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("d", [64, 99])
@pytest.mark.parametrize("f32", [False, True])
def test_accumulate_at_any_alignment(f32, d, off):
    from paper_2609_20359_b200.head import Head
    n, V = 70, 600
    h, w, y, _ = make(n, V, d)
    dtype = torch.float32 if f32 else torch.bfloat16
    gw = torch.empty(V * d + off, dtype=dtype, device=DEV)[off:].view(V, d)
    gw.copy_(torch.randn(V, d, device=DEV))
    before = gw.double()
    live = torch.ones(n, dtype=torch.bool, device=DEV)
    Head(n, V, d, grad_dtype="f32" if f32 else "bf16").xent_step(h, w, y, grad_weight=gw, accumulate=True)
    ref = R.with_gradients(h, w, lambda z: (*R.xent_rows(z, y, live, 0.0, 0.0), live))
    ref["grad_weight"] = ref["grad_weight"] + before
    R.check_grads(ref, grad_weight=gw)


def test_a_list_that_is_the_whole_vocabulary():
    """Nothing is outside the list: the tail class is empty and both readings of the tail agree."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 7, 64, 64
    h, w, y, g = make(n, V, d)
    idx, t = teacher(n, V, V, g, ragged=False)
    head = Head(n, V, d, top=V)
    out = []
    for tl in (None, torch.logsumexp(t.double(), 1).float()):
        gh, gw = buffers(n, V, d)
        loss, _ = head.distill_step(h, w, idx, t, gh, gw, teacher_lse=tl)
        out.append((loss.double(), gh.double()))
    # teacher_lse is rounded to fp32: q is off by 2^-23 |lse|, the loss by that times its logarithms
    assert bool(torch.isfinite(out[1][0]).all()) and bool(((out[0][0] - out[1][0]).abs() <= 1e-5 * (1 + out[0][0])).all())
    assert bool(((out[0][1] - out[1][1]).abs() <= 2.0 ** -7 * out[0][1].abs() + 1e-5).all())


def test_offsets_beyond_32_bits():
    """A weight and its gradient of more than 2^31 elements; labels at both ends of the vocabulary."""
    from paper_2609_20359_b200.head import Head
    n, V, d = 4, 1_100_003, 2048
    g = torch.Generator(device=DEV).manual_seed(0)
    w = torch.empty(V, d, dtype=torch.bfloat16, device=DEV)
    for lo in range(0, V, 1 << 17):
        w[lo: lo + (1 << 17)] = torch.randn(min(1 << 17, V - lo), d, generator=g, device=DEV) / 30
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    y = torch.tensor([0, V - 1, V - 200, 1_050_000], device=DEV)
    gh, gw = buffers(n, V, d)
    loss, lse = Head(n, V, d).xent_step(h, w, y, gh, gw, row_weight=torch.ones(n, device=DEV))
    z = torch.cat([h.double() @ w[lo: lo + (1 << 16)].double().t() for lo in range(0, V, 1 << 16)], 1)
    p = torch.softmax(z, 1)
    p[torch.arange(n), y] -= 1
    want = torch.logsumexp(z, 1)
    assert bool(((lse.double() - want).abs() <= 1e-5).all())
    assert bool(((loss.double() - (want - z.gather(1, y[:, None])[:, 0])).abs() <= 2e-5).all())
    for lo in (0, 524288, 1_048_576, V - 3000):
        part = p[:, lo: lo + 3000].t() @ h.double()
        bound = p[:, lo: lo + 3000].abs().t() @ h.double().abs() * (2.0 ** -8 + 2e-5) + 2.0 ** -8 * part.abs() + 1e-30
        assert bool(((gw[lo: lo + 3000].double() - part).abs() <= bound).all()), lo
    assert not bool(torch.isnan(gw[::997]).any())
    dh = sum(p[:, lo: lo + (1 << 16)] @ w[lo: lo + (1 << 16)].double() for lo in range(0, V, 1 << 16))
    size = sum(p[:, lo: lo + (1 << 16)].abs() @ w[lo: lo + (1 << 16)].double().abs() for lo in range(0, V, 1 << 16))
    assert bool(((gh.double() - dh).abs() <= size * (2.0 ** -8 + 2e-5 + V / 16 * 2.0 ** -23) + 2.0 ** -8 * dh.abs()).all())


def test_bounded_waits_run_out():
    """Nothing announces the operands: every wait of the kernels gives up, the status word says so, the next call is right."""
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.head import Head
    n, V, d = 300, 2000, 256
    h, w, y, _ = make(n, V, d)
    head = Head(n, V, d)
    gh, gw = buffers(n, V, d)
    want = [t.clone() for t in (*head.xent_step(h, w, y, gh, gw), gh, gw)]
    assert head.status() == 0
    fls.fls_debug_expire_next_head_wait(head.handle, 200)
    head.xent_step(h, w, y, gh, gw)
    assert head.status() == fls.FLS_STATUS_WAIT_EXPIRED
    got = (*head.xent_step(h, w, y, gh, gw), gh, gw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_no_rows():
    from paper_2609_20359_b200.head import Head
    V, d = 300, 64
    h, w, y, _ = make(0, V, d)
    head = Head(16, V, d)
    gh, gw = buffers(0, V, d)
    loss, lse = head.xent_step(h, w, y, gh, gw)
    assert loss.shape == lse.shape == (0,) and not bool(gw.any())
    gw.fill_(2.0)
    head.xent_step(h, w, y, gh, gw, accumulate=True)
    assert bool((gw == 2.0).all())


def test_example_trains():
    """Loss, gradients into the plan's buffers, optimizer, averaging and distillation together."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "federated_head.py")
    spec = importlib.util.spec_from_file_location("federated_head", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    history, taught = mod.main(quiet=True)
    assert history[0] > math.log(mod.VOCAB) - 1 and history[-1] < 0.6 * history[0]
    assert all(math.isfinite(x) for x in taught) and taught[-1] < 0.6 * taught[0]
