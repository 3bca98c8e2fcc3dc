"""Random sizes, types, strides, alignments and token distributions of the embedding and the norms against 64 bits."""
import math
import random

import pytest
import torch

from tests import layers_reference as R
from tests.test_embed_gpu import DEV, TYPES, embedding, gen, outside, rows, tokens_of
from tests.test_norm_large_batches import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


def spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def width(rng, hi):
    d = spread(rng, 1, hi)
    return (d + 7) // 8 * 8 if rng.random() < 0.6 else d


@pytest.mark.parametrize("seed", range(150))
def test_embedding(seed):
    rng = random.Random(seed)
    g = gen(seed)
    d, pad, shift = width(rng, 5000), rng.choice([0, 0, 8, 3]), rng.choice([0, 0, 8, 1])
    n = max(1, min(spread(rng, 1, 300000), 20_000_000 // d))
    V = max(1, min(spread(rng, 1, 200000), 20_000_000 // d))
    act, grad = rng.choice(["bf16", "f32"]), rng.choice(["bf16", "f32"])
    tok = tokens_of(rng.choice(["random", "text", "text", "same", "few", "falling", "mixed", "ignored"]), n, V, g)
    dy, _ = rows(n, d, TYPES[act], g, pad, shift)
    gw, flat = rows(V, d, TYPES[grad], g, pad, shift)
    e = embedding(n, V, d, act_dtype=act, grad_dtype=grad)
    e.workspace.memory.fill_(255)
    gw.fill_(float("nan"))
    e.grad(tok, dy, gw, scale=1.3)
    R.check_embed_grad(gw, tok, dy, scale=1.3)
    old = torch.randn(V, d, generator=g, device=DEV).to(TYPES[grad])
    gw.copy_(old)
    e.grad(tok, dy, gw, accumulate=True)
    R.check_embed_grad(gw, tok, dy, old=old)
    assert bool(outside(flat, gw).isnan().all())
    w, _ = rows(V, d, torch.bfloat16, g, pad, shift)
    got, want = e.lookup(tok, w, scale=0.7), R.lookup(tok, w, 0.7, -100, TYPES[act])
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


@pytest.mark.parametrize("seed", range(150))
def test_norm(seed):
    rng = random.Random(1000 + seed)
    d = width(rng, 20000 if rng.random() < 0.2 else 5000)
    n = max(1, min(spread(rng, 1, 100000), 10_000_000 // d))
    x, y, w, grad = (rng.choice(["bf16", "f32"]) for _ in range(4))
    run(n, d, rng.choice(["layer", "rms"]), x, y, w, grad, rng.random() < 0.5, rng.choice([0, 0, 8, 3]), rng.choice([0, 0, 8, 1]),
        rng.choice([0, 0, 0, 1, 8]), gen(seed))
