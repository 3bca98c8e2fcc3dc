"""What the two gradients of a head's step owe each other, and where they end."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_2609_20359_b200 import build
    build.build()


def make(n, V, d, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(n, d, generator=g, device=DEV).bfloat16()
    w = (torch.randn(V, d, generator=g, device=DEV) * (2.0 / math.sqrt(d))).bfloat16()
    y = torch.randint(0, V, (n,), generator=g, device=DEV)
    return h, w, y


# formed in several pieces, kept in part, kept altogether, one piece; calls of all rows and of fewer than the head was made for
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("rows,n,V,d,piece", [(400, 400, 6000, 256, 1 << 20), (700, 700, 2500, 320, 1 << 20), (300, 300, 3000, 904, 1 << 22),
                                              (130, 130, 20000, 1024, 0), (64, 64, 40000, 64, 1 << 22), (2000, 700, 9000, 512, 1 << 24)])
def test_one_gradient_alone_has_the_bits_of_both(rows, n, V, d, piece, f32):
    from paper_2609_20359_b200.head import Head
    h, w, y = make(n, V, d)
    head = Head(rows, V, d, grad_dtype="f32" if f32 else "bf16", piece_bytes=piece)

    def buffers():
        return (torch.full((n, d), math.nan, dtype=torch.bfloat16, device=DEV),
                torch.full((V, d), math.nan, dtype=head.grad_torch_dtype, device=DEV))

    both, alone = buffers(), buffers()
    head.xent_step(h, w, y, *both)
    head.xent_step(h, w, y, grad_hidden=alone[0])
    head.xent_step(h, w, y, grad_weight=alone[1])
    assert torch.equal(alone[0], both[0]) and torch.equal(alone[1], both[1])
