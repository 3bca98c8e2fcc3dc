"""A Norm that is made while a graph is being captured: its workspace is cleared by the graph alone, which may not have been
replayed when the object is used elsewhere."""
import pytest
import torch

from tests import layers_reference as R
from tests.test_embed_gpu import DEV, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2609_20359_b200 import build
    build.build()


@pytest.mark.parametrize("use", ["eager", "another stream", "another graph", "replay"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_used_before_the_graph_is_replayed(kind, use):
    from paper_2609_20359_b200.norm import Norm
    n, d, g = 100, 768, gen(9)                              # so few that the last CTA adds the weight gradients up
    x, dy = (torch.randn(n, d, generator=g, device=DEV).bfloat16() for _ in range(2))
    w = torch.randn(d, generator=g, device=DEV).bfloat16()
    first = Norm(n, d, kind, grad_dtype="f32", device=DEV)
    _, mean, rstd = first.forward(x, w)
    dw, db = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    first.backward(x, w, mean, rstd, dy, dw, db)
    # what the captured object's memory holds: the ones that another graph left there
    pool = torch.cuda.graph_pool_handle()
    before, graph, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(before, pool=pool):
        junk = torch.empty(first.workspace.memory.numel(), dtype=torch.uint8, device=DEV)
        junk.fill_(255)
    before.replay()
    torch.cuda.synchronize()
    at = junk.data_ptr()
    del junk

    with torch.cuda.graph(graph, pool=pool):
        op = Norm(n, d, kind, grad_dtype="f32", device=DEV)
        dx = op.backward(x, w, mean, rstd, dy, dw, db)
    assert op.workspace.memory.data_ptr() == at
    for t in (dw, db):
        t.fill_(float("nan"))
    if use == "eager":
        dx = op.backward(x, w, mean, rstd, dy, dw, db)
    elif use == "another stream":
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        dx = op.backward(x, w, mean, rstd, dy, dw, db, stream=s.cuda_stream)
        torch.cuda.current_stream().wait_stream(s)
    elif use == "another graph":
        with torch.cuda.graph(other):
            dx = op.backward(x, w, mean, rstd, dy, dw, db)
        other.replay()
    else:
        graph.replay()
    R.check_backward(x, w, mean, rstd, dy, None, dx, dw, db)
    # and in turn
    for again in (graph.replay, lambda: op.backward(x, w, mean, rstd, dy, dw, db), graph.replay):
        for t in (dw, db):
            t.fill_(float("nan"))
        again()
        R.check_backward(x, w, mean, rstd, dy, None, None, dw, db)
    torch.cuda.synchronize()
    del graph, other, before
