"""Norm: layer norm and root mean square norm on libfls (device memory and streams only).

All arithmetic happens in libfls through the fls_norm_* calls; this class owns one handle and its workspace, and checks the
tensors it is given.
"""
from __future__ import annotations

import torch

from . import _binding as fls
from .workspace import Arguments, Workspace, device_of, dtype_of, matrix, vector


class Norm:
    """Norm of rows of `dim` values, with the residual addition before it on request, and its gradients.

    max_rows: N of the largest call.  kind: "layer" or "rms".  Types, each "bf16" or "f32": x_dtype of the rows, the residual,
    their sum and its gradients; y_dtype of the result and its gradient; weight_dtype of weight and bias; grad_dtype of their
    gradients (as `Session`'s gradient buffers, whose units they may be written into).  grads=False: forward passes only.

    Every call is enqueued on `stream` (default: torch's current stream) and returns without waiting.  Forward passes may be made
    on several streams and from several host threads at once.  Backward passes use the workspace, one call at a time: those of
    one Norm belong on one stream, or on streams ordered by events.  A Norm may be dropped while its calls run (a stream given
    by its handle has to outlive it); a captured graph has to be dropped first.
    """

    def __init__(self, max_rows: int, dim: int, kind: str = "layer", eps: float = 1e-5, x_dtype: str = "bf16", y_dtype: str = "bf16",
                 weight_dtype: str = "bf16", grad_dtype: str = "bf16", grads: bool = True, device: str = "cuda:0"):
        self.handle = None
        if kind not in ("layer", "rms"):
            raise ValueError("kind must be 'layer' or 'rms'")
        self.device = device_of(device)
        self.x_torch_dtype, x = dtype_of(x_dtype, "x_dtype")
        self.y_torch_dtype, y = dtype_of(y_dtype, "y_dtype")
        self.weight_torch_dtype, w = dtype_of(weight_dtype, "weight_dtype")
        self.grad_torch_dtype, g = dtype_of(grad_dtype, "grad_dtype")
        self.max_rows, self.dim, self.kind, self.eps, self.grads = max_rows, dim, kind, eps, grads
        self.handle = fls.fls_norm_create(max_rows, dim, fls.FLS_NORM_RMS if kind == "rms" else fls.FLS_NORM_LAYER, eps, x, y, w, g, grads)
        self.workspace = Workspace(fls.fls_norm_query(self.handle)["workspace_bytes"], self.device)
        mem = self.workspace.memory
        self._args = Arguments(forward=(fls.fls_norm_io, {}),
                               backward=(fls.fls_norm_grad_io, dict(workspace=mem.data_ptr(), workspace_bytes=mem.numel())))

    # ------------------------------------------------------------------ calls
    def forward(self, x, weight=None, bias=None, y=None, stats: bool = True, stream=None):
        """(y, mean, rstd): the norm of every row of x.  mean and rstd (fp32, what backward takes) are None without stats, and
        mean for a root mean square norm."""
        y, _, mean, rstd = self._forward(x, None, weight, bias, y, None, stats, stream)
        return y, mean, rstd

    def add_forward(self, x, residual, weight=None, bias=None, y=None, total=None, stats: bool = True, stream=None):
        """(y, total, mean, rstd): total = x + residual, rounded to their type, and the norm of its rows.  `total` may be x or
        residual itself."""
        return self._forward(x, residual, weight, bias, y, total, stats, stream)

    def backward(self, x, weight, mean, rstd, grad_y, grad_weight=None, grad_bias=None, grad_total=None, grad_x=None,
                 input_grad: bool = True, accumulate: bool = False, stream=None):
        """grad_x, the gradient of what was normalised (`x`: total, after add_forward), plus grad_total if given; the gradients of
        weight and bias go to grad_weight and grad_bias, each optional, accumulate adds to them.  `grad_x` may be grad_total
        itself; input_grad=False leaves it out."""
        args, dim, xt, gt = self._args, self.dim, self.x_torch_dtype, self.grad_torch_dtype
        io = args.backward
        io.x, io.x_stride = matrix(x, "x", None, dim, xt)
        n = io.rows = x.shape[0]
        io.weight = vector(weight, "weight", dim, self.weight_torch_dtype)
        if (mean is None) != (self.kind == "rms"):
            raise ValueError("mean belongs to layer norms, and to all of them")
        io.mean = vector(mean, "mean", n, torch.float32)
        if rstd is None:
            raise ValueError("rstd is needed")
        io.rstd = vector(rstd, "rstd", n, torch.float32)
        io.grad_y, io.grad_y_stride = matrix(grad_y, "grad_y", n, dim, self.y_torch_dtype)
        if not input_grad:
            if grad_x is not None or grad_total is not None:
                raise ValueError("grad_x and grad_total without input_grad")
            io.grad_x, io.grad_x_stride = None, 0
        elif grad_x is None:
            grad_x = torch.empty_like(x) if stream is None else self.workspace.new(stream, (n, dim), xt)
            io.grad_x, io.grad_x_stride = grad_x.data_ptr(), 0
        else:
            io.grad_x, io.grad_x_stride = matrix(grad_x, "grad_x", n, dim, xt)
        io.grad_total, io.grad_total_stride = (None, 0) if grad_total is None else matrix(grad_total, "grad_total", n, dim, xt)
        io.grad_weight = vector(grad_weight, "grad_weight", dim, gt)
        io.grad_bias = vector(grad_bias, "grad_bias", dim, gt)
        io.accumulate = accumulate
        fls._check(fls.lib.fls_norm_backward(self.handle, args.backward_ref, self.workspace.use(stream)))
        return grad_x

    def _forward(self, x, residual, weight, bias, y, total, stats, stream):
        args, dim, xt, yt, new = self._args, self.dim, self.x_torch_dtype, self.y_torch_dtype, self.workspace.new
        io = args.forward
        io.x, io.x_stride = matrix(x, "x", None, dim, xt)
        n = io.rows = x.shape[0]
        io.weight = vector(weight, "weight", dim, self.weight_torch_dtype)
        io.bias = vector(bias, "bias", dim, self.weight_torch_dtype)
        if residual is None:
            io.residual = io.total = None
            io.residual_stride = io.total_stride = 0
        else:
            io.residual, io.residual_stride = matrix(residual, "residual", n, dim, xt)
            if total is None:
                total = torch.empty_like(x) if stream is None else new(stream, (n, dim), xt)
                io.total, io.total_stride = total.data_ptr(), 0
            else:
                io.total, io.total_stride = matrix(total, "total", n, dim, xt)
        if y is None:
            y = torch.empty_like(x) if stream is None and xt is yt else new(stream, (n, dim), yt)
            io.y, io.y_stride = y.data_ptr(), 0
        else:
            io.y, io.y_stride = matrix(y, "y", n, dim, yt)
        mean = rstd = io.mean = io.rstd = None
        if stats:
            if self.kind == "layer":
                mean = new(stream, n, torch.float32)
                io.mean = mean.data_ptr()
            rstd = new(stream, n, torch.float32)
            io.rstd = rstd.data_ptr()
        fls._check(fls.lib.fls_norm_forward(self.handle, args.forward_ref, self.workspace.stream(stream)))
        return y, total, mean, rstd

    def close(self) -> None:
        if self.handle is not None:
            fls.fls_norm_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
