"""Calls of one Embedding or Norm from two host threads at once."""
import threading

import pytest
import torch


class Gate:
    """Stands in for the library: a call of `name` waits inside for the other thread's, then writes down what it was given."""

    def __init__(self, lib, name, fields):
        self.lib, self.name, self.fields = lib, name, fields
        self.both, self.seen = threading.Barrier(2), {}

    def __getattr__(self, name):
        return self._call if name == self.name else getattr(self.lib, name)

    def _call(self, handle, ref, stream):
        self.both.wait(20)                                  # both calls are prepared
        self.seen[threading.get_ident()] = {f: getattr(ref._obj, f) for f in self.fields}
        self.both.wait(20)
        return 0


class Memory:
    """A workspace on the host."""

    def __init__(self, nbytes, device):
        self.memory = torch.zeros(max(nbytes, 1), dtype=torch.uint8)

    def stream(self, stream):
        return 0

    use = stream

    def new(self, stream, shape, dtype):
        return torch.empty(shape, dtype=dtype)


@pytest.fixture
def host(monkeypatch):
    """The classes without a device: only the preparation of calls is theirs here."""
    from paper_2609_20359_b200 import build
    build.build()
    from paper_2609_20359_b200 import embed, norm
    for m in (embed, norm):
        monkeypatch.setattr(m, "device_of", lambda device: torch.device("cpu"))
        monkeypatch.setattr(m, "Workspace", Memory)
        monkeypatch.setattr(m, "matrix", lambda t, name, rows, cols, dtype: (t.data_ptr(), 0))
        monkeypatch.setattr(m, "vector", lambda t, name, n, dtype: None if t is None else t.data_ptr())
    return monkeypatch


def together(calls):
    """What each of two threads' calls returns."""
    got, errors = [None, None], []

    def work(k):
        try:
            got[k] = (threading.get_ident(), calls[k]())
        except Exception as e:                              # shown by the test's thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not errors, errors
    return got


def test_lookups_keep_their_own_arguments(host):
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.embed import Embedding
    e = Embedding(100, 50, 16, grads=False)
    gate = Gate(fls.lib, "fls_embed_lookup", ["tokens", "token", "weight", "out", "scale", "ignore_token"])
    host.setattr(fls, "lib", gate)
    toks = [torch.zeros(n, dtype=torch.int64) for n in (100, 3)]
    tables = [torch.zeros(50, 16, dtype=torch.bfloat16) for _ in range(2)]
    got = together([lambda k=k: e.lookup(toks[k], tables[k], scale=float(k + 2), ignore_token=-k) for k in range(2)])
    for k, (thread, out) in enumerate(got):
        assert gate.seen[thread] == dict(tokens=len(toks[k]), token=toks[k].data_ptr(), weight=tables[k].data_ptr(), out=out.data_ptr(),
                                         scale=float(k + 2), ignore_token=-k)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_forward_passes_keep_their_own_arguments(host, kind):
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.norm import Norm
    op = Norm(100, 16, kind, grads=False)
    gate = Gate(fls.lib, "fls_norm_forward", ["rows", "x", "residual", "weight", "y", "total", "mean", "rstd"])
    host.setattr(fls, "lib", gate)
    x, r = ([torch.zeros(n, 16, dtype=torch.bfloat16) for n in (100, 3)] for _ in range(2))
    w = [torch.zeros(16, dtype=torch.bfloat16) for _ in range(2)]
    calls = [lambda: op.add_forward(x[0], r[0], w[0]), lambda: op.forward(x[1], w[1])]
    (first, (y0, total, mean0, rstd0)), (second, (y1, mean1, rstd1)) = together(calls)
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    assert gate.seen[first] == dict(rows=100, x=at(x[0]), residual=at(r[0]), weight=at(w[0]), y=at(y0), total=at(total), mean=at(mean0),
                                    rstd=at(rstd0))
    assert gate.seen[second] == dict(rows=3, x=at(x[1]), residual=None, weight=at(w[1]), y=at(y1), total=None, mean=at(mean1), rstd=at(rstd1))


def test_gradients_keep_their_own_arguments(host):
    """Gradients share the workspace, so their work is ordered by streams and events; what a call is given is its own all the same."""
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.norm import Norm
    e, op = Embedding(100, 50, 16), Norm(100, 16, "rms")
    lib = fls.lib
    gate = Gate(lib, "fls_embed_grad", ["tokens", "grad_out", "grad_weight", "accumulate", "workspace"])
    host.setattr(fls, "lib", gate)
    toks = [torch.zeros(n, dtype=torch.int64) for n in (100, 3)]
    dy = [torch.zeros(n, 16, dtype=torch.bfloat16) for n in (100, 3)]
    gw = [torch.zeros(50, 16, dtype=torch.bfloat16) for _ in range(2)]
    got = together([lambda k=k: e.grad(toks[k], dy[k], gw[k], accumulate=bool(k)) for k in range(2)])
    for k, (thread, _) in enumerate(got):
        assert gate.seen[thread] == dict(tokens=len(toks[k]), grad_out=dy[k].data_ptr(), grad_weight=gw[k].data_ptr(), accumulate=k,
                                         workspace=e.workspace.memory.data_ptr())
    gate = Gate(lib, "fls_norm_backward", ["rows", "x", "grad_y", "grad_x", "rstd", "workspace"])
    host.setattr(fls, "lib", gate)
    x, rstd = [torch.zeros_like(t) for t in dy], [torch.zeros(n) for n in (100, 3)]
    got = together([lambda k=k: op.backward(x[k], None, None, rstd[k], dy[k]) for k in range(2)])
    for k, (thread, dx) in enumerate(got):
        assert gate.seen[thread] == dict(rows=len(dy[k]), x=x[k].data_ptr(), grad_y=dy[k].data_ptr(), grad_x=dx.data_ptr(),
                                         rstd=rstd[k].data_ptr(), workspace=op.workspace.memory.data_ptr())


@pytest.mark.gpu
def test_forward_passes_from_two_threads():
    """Two threads, each on a stream of its own, calls of different sizes of one object."""
    from paper_2609_20359_b200 import _binding as fls
    from paper_2609_20359_b200.embed import Embedding
    from paper_2609_20359_b200.norm import Norm
    dev, V, d, sizes, calls = "cuda:0", 500, 256, (300, 7), 400
    g = torch.Generator(device=dev).manual_seed(8)
    table = torch.randn(V, d, generator=g, device=dev).bfloat16()
    toks = [torch.randint(0, V, (n,), generator=g, device=dev) for n in sizes]
    emb, norm = Embedding(max(sizes), V, d, grads=False), Norm(max(sizes), d, "rms", grads=False)
    want = [norm.add_forward(emb.lookup(t, table, scale=k + 1.0), emb.lookup(t.flip(0), table)) for k, t in enumerate(toks)]
    torch.cuda.synchronize()
    launches = fls.fls_embed_get_launch_count(emb.handle), fls.fls_norm_get_launch_count(norm.handle)

    def work(k):
        torch.cuda.set_device(dev)
        bad, s = 0, torch.cuda.Stream()
        with torch.cuda.stream(s):
            flipped = toks[k].flip(0)
            for _ in range(calls):
                out = norm.add_forward(emb.lookup(toks[k], table, scale=k + 1.0), emb.lookup(flipped, table))
                bad += sum(int(not torch.equal(a, b)) for a, b in zip(out, want[k]) if a is not None)
            s.synchronize()
        return bad

    got = together([lambda k=k: work(k) for k in range(2)])
    assert [bad for _, bad in got] == [0, 0]
    assert fls.fls_embed_get_launch_count(emb.handle) - launches[0] == 4 * calls
    assert fls.fls_norm_get_launch_count(norm.handle) - launches[1] == 2 * calls
