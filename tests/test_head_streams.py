"""A Head's workspace on other streams than the one it was made on: ordered with the clear at its start, and not handed to
another tensor before the last call is done."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N, V, D = 300, 4000, 256
BUSY = 200_000_000                                    # clock cycles, about a tenth of a second


@pytest.fixture(scope="module")
def case():
    """Inputs and, computed in peace, what every call has to give."""
    from paper_2609_20359_b200 import build
    build.build()
    from paper_2609_20359_b200.head import Head
    g = torch.Generator(device=DEV).manual_seed(0)
    h = torch.randn(N, D, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, D, generator=g, device=DEV) / 8).bfloat16()
    y = torch.randint(0, V, (N,), generator=g, device=DEV)
    gh, gw = torch.empty_like(h), torch.empty_like(w)
    loss, lse = Head(N, V, D).xent_step(h, w, y, gh, gw)
    torch.cuda.synchronize()
    return (h, w, y), (loss, lse, gh, gw)


def outputs():
    gh = torch.full((N, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    gw = torch.full((V, D), float("nan"), dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    return gh, gw


def step(head, inputs, gh, gw, stream, how):
    if how == "current":
        with torch.cuda.stream(stream):
            return head.xent_step(*inputs, gh, gw)
    return head.xent_step(*inputs, gh, gw, stream=stream if how == "stream" else stream.cuda_stream)


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_first_call_while_the_constructors_stream_is_busy(case, how):
    from paper_2609_20359_b200.head import Head
    inputs, want = case
    gh, gw = outputs()
    s = torch.cuda.Stream()
    torch.cuda._sleep(BUSY)
    head = Head(N, V, D)
    loss, lse = step(head, inputs, gh, gw, s, how)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, gh, gw)))
    assert head.status() == 0 and int(head.rows_taking_part()) == N


@pytest.mark.parametrize("how", ["stream", "handle", "current"])
def test_dropped_while_its_call_is_waiting(case, how):
    from paper_2609_20359_b200.head import Head
    inputs, want = case
    gh, gw = outputs()
    s = torch.cuda.Stream()
    head = Head(N, V, D)
    size, address = head.workspace.numel(), head.workspace.data_ptr()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    loss, lse = step(head, inputs, gh, gw, s, how)
    del head
    junk = torch.empty(size, dtype=torch.uint8, device=DEV)
    assert junk.data_ptr() + size <= address or address + size <= junk.data_ptr()
    junk.fill_(255)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, gh, gw)))


def test_made_on_a_side_stream_and_used_on_the_default_one(case):
    from paper_2609_20359_b200.head import Head
    inputs, want = case
    gh, gw = outputs()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
        head = Head(N, V, D)
    loss, lse = head.xent_step(*inputs, gh, gw)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, gh, gw)))
