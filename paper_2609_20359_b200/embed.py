"""Embedding: the input end of a language model on libfls (device memory and streams only).

All arithmetic happens in libfls through the fls_embed_* calls; this class owns one handle and its workspace, and checks the
tensors it is given.
"""
from __future__ import annotations

import torch

from . import _binding as fls
from .workspace import Arguments, Workspace, device_of, dtype_of, matrix, vector


class Embedding:
    """Rows of a [vocab, dim] bf16 table by token, and the gradient of that table.

    max_tokens, vocab, dim: N of the largest call, V and d.  act_dtype: "bf16" or "f32", the type of looked-up rows and of
    their gradients.  grad_dtype: the type of the table's gradient (as `Session`'s gradient buffers, whose units it may be
    written into).  grads=False: lookups only.

    Every call is enqueued on `stream` (default: torch's current stream) and returns without waiting.  Lookups may be made on
    several streams and from several host threads at once.  Gradients use the workspace, one call at a time: those of one
    Embedding belong on one stream, or on streams ordered by events.  An Embedding may be dropped while its calls run (a stream
    given by its handle has to outlive it); a captured graph has to be dropped first.
    """

    def __init__(self, max_tokens: int, vocab: int, dim: int, act_dtype: str = "bf16", grad_dtype: str = "bf16", grads: bool = True,
                 device: str = "cuda:0"):
        self.handle = None
        self.device = device_of(device)
        self.act_torch_dtype, act = dtype_of(act_dtype, "act_dtype")
        self.grad_torch_dtype, grad = dtype_of(grad_dtype, "grad_dtype")
        self.max_tokens, self.vocab, self.dim, self.grads = max_tokens, vocab, dim, grads
        self.handle = fls.fls_embed_create(max_tokens, vocab, dim, grads, act, grad)
        self.workspace = Workspace(fls.fls_embed_query(self.handle)["workspace_bytes"], self.device)
        mem = self.workspace.memory
        # apart, since the library looks at all strides of a structure, and a refused call's must not be in the way of the other's
        self._args = Arguments(lookup=(fls.fls_embed_io, {}),
                               grad=(fls.fls_embed_io, dict(workspace=mem.data_ptr(), workspace_bytes=mem.numel())))

    def lookup(self, tokens, weight, out=None, scale: float = 1.0, ignore_token: int = -100, stream=None):
        """scale * weight[tokens], [N, dim]: zeros where a token is ignore_token, NaN where it is outside the table."""
        args = self._args
        io = args.lookup
        n = self._tokens(io, tokens)
        io.weight, io.weight_stride = matrix(weight, "weight", self.vocab, self.dim, torch.bfloat16)
        if out is None:
            out = self.workspace.new(stream, (n, self.dim), self.act_torch_dtype)
            io.out, io.out_stride = out.data_ptr(), 0
        else:
            io.out, io.out_stride = matrix(out, "out", n, self.dim, self.act_torch_dtype)
        io.scale, io.ignore_token = scale, ignore_token
        fls._check(fls.lib.fls_embed_lookup(self.handle, args.lookup_ref, self.workspace.stream(stream)))
        return out

    def grad(self, tokens, grad_out, grad_weight, scale: float = 1.0, accumulate: bool = False, ignore_token: int = -100,
             stream=None) -> None:
        """grad_weight [vocab, dim] becomes (accumulate: is added) scale times the sums of the rows of grad_out by token."""
        args = self._args
        io = args.grad
        n = self._tokens(io, tokens)
        io.grad_out, io.grad_out_stride = matrix(grad_out, "grad_out", n, self.dim, self.act_torch_dtype)
        io.grad_weight, io.grad_weight_stride = matrix(grad_weight, "grad_weight", self.vocab, self.dim, self.grad_torch_dtype)
        io.scale, io.ignore_token, io.accumulate = scale, ignore_token, accumulate
        fls._check(fls.lib.fls_embed_grad(self.handle, args.grad_ref, self.workspace.use(stream)))

    @staticmethod
    def _tokens(io, tokens) -> int:
        n = tokens.numel()
        io.token = vector(tokens, "tokens", n, torch.int64)
        io.tokens = n
        return n

    def close(self) -> None:
        if self.handle is not None:
            fls.fls_embed_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
