"""Head: the loss end of a language model on libfls (device memory and streams only).

All arithmetic happens in libfls through the fls_head_* calls; this class owns one head handle, its workspace and the
outputs, and checks the tensors it is given.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import _binding as fls


def _matrix(t: torch.Tensor, name: str, rows: Optional[int], cols: int, dtype: torch.dtype, device: torch.device):
    """Checks a 2-D tensor whose rows are contiguous; returns (address, elements between rows)."""
    shape = t.shape
    if len(shape) != 2 or shape[1] != cols or (rows is not None and shape[0] != rows) or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor of shape [{'N' if rows is None else rows}, {cols}] on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    row, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous (stride {one})")
    if shape[0] <= 1:
        row = cols
    elif row < cols:
        raise ValueError(f"{name}: rows overlap (stride {row})")
    return t.data_ptr(), row


def _dense(t: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype, device: torch.device):
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _empty_on(stream, shape, dtype: torch.dtype, device: torch.device) -> torch.Tensor:
    """Memory whose reuse is ordered by the stream that writes it, which need not be torch's current one."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream):
        return torch.empty(shape, dtype=dtype, device=device)


class Head:
    """Losses of a linear head without kept logits.

    max_rows, vocab, dim: N of the largest call, V and d.  top: teacher entries per row (0: no distillation).
    grad_dtype: "bf16" or "f32", the type of weight gradients (as `Session`'s gradient buffers, whose units they may be
    written into).  grads=False: a workspace for losses only.  any_weight: accept weights of any alignment and stride.

    Every call is enqueued on `stream` (default: torch's current stream) and returns without waiting; the constructor waits
    until the workspace is cleared.  The workspace is used by one call at a time: calls of one Head belong on one stream, or on
    streams ordered by events.  A Head may be dropped while its calls run (a stream given by its handle has to outlive it); a
    captured graph has to be dropped first.
    """

    def __init__(self, max_rows: int, vocab: int, dim: int, top: int = 0, grad_dtype: str = "bf16", grads: bool = True,
                 any_weight: bool = False, piece_bytes: int = 0, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("libfls needs a CUDA device; there is no CPU path")
        if grad_dtype not in ("bf16", "f32"):
            raise ValueError("grad_dtype must be 'bf16' or 'f32'")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        torch.cuda.set_device(self.device)
        self.max_rows, self.vocab, self.dim, self.top = max_rows, vocab, dim, top
        self.grad_torch_dtype = torch.float32 if grad_dtype == "f32" else torch.bfloat16
        self.handle = None
        self.handle = fls.fls_head_create(max_rows, vocab, dim, top, grads, fls.FLS_GRAD_F32 if grad_dtype == "f32" else fls.FLS_GRAD_BF16,
                                          any_weight, piece_bytes)
        self.layout = fls.fls_head_query(self.handle)
        self.workspace = torch.empty(self.layout["workspace_bytes"], dtype=torch.uint8, device=self.device)
        self.workspace[:256].zero_()
        # The first call may be on any stream: the clear, and what used this memory before, must not come after it.
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(self.device).synchronize()
        self._streams = {fls._stream_handle(None)}             # those that torch's allocator knows to use the workspace
        self._args = fls.fls_head_io(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace.numel())   # of the call in preparation

    # ------------------------------------------------------------------ calls
    def xent(self, hidden, weight, labels, ignore_label: int = -100, label_smoothing: float = 0.0, z_loss: float = 0.0, stream=None):
        """(loss, lse) of every row, fp32."""
        io, out = self._io(hidden, weight, labels, ignore_label, None, None, None, False, stream)
        fls.fls_head_xent(self.handle, io, label_smoothing, z_loss, self._use(stream))
        return out

    def xent_step(self, hidden, weight, labels, grad_hidden=None, grad_weight=None, row_weight=None, accumulate: bool = False,
                  ignore_label: int = -100, label_smoothing: float = 0.0, z_loss: float = 0.0, stream=None):
        """(loss, lse); the gradients of sum(row_weight * loss) (default: the mean over the rows that take part) are written
        to grad_hidden (bf16) and grad_weight, each optional; accumulate adds to grad_weight."""
        io, out = self._io(hidden, weight, labels, ignore_label, grad_hidden, grad_weight, row_weight, accumulate, stream)
        fls.fls_head_xent(self.handle, io, label_smoothing, z_loss, self._use(stream))
        return out

    def distill(self, hidden, weight, top_index, top_logit, labels=None, teacher_lse=None, temperature: float = 1.0,
                distill_weight: float = 1.0, label_weight: float = 0.0, ignore_label: int = -100, stream=None):
        """(loss, lse) against a teacher's top logits; teacher_lse given: what is outside the list counts as one class."""
        return self._distill(hidden, weight, top_index, top_logit, labels, teacher_lse, temperature, distill_weight, label_weight,
                             ignore_label, None, None, None, False, stream)

    def distill_step(self, hidden, weight, top_index, top_logit, grad_hidden=None, grad_weight=None, row_weight=None,
                     accumulate: bool = False, labels=None, teacher_lse=None, temperature: float = 1.0, distill_weight: float = 1.0,
                     label_weight: float = 0.0, ignore_label: int = -100, stream=None):
        """As distill, with gradients as in xent_step."""
        return self._distill(hidden, weight, top_index, top_logit, labels, teacher_lse, temperature, distill_weight, label_weight,
                             ignore_label, grad_hidden, grad_weight, row_weight, accumulate, stream)

    def _distill(self, hidden, weight, top_index, top_logit, labels, teacher_lse, temperature, distill_weight, label_weight,
                 ignore_label, grad_hidden, grad_weight, row_weight, accumulate, stream):
        if label_weight and labels is None:
            raise ValueError("label_weight needs labels")
        io, out = self._io(hidden, weight, labels if label_weight else None, ignore_label, grad_hidden, grad_weight, row_weight, accumulate,
                            stream)
        n = io.rows
        t = fls.fls_distill_desc(_dense(top_index, "top_index", (n, self.top), torch.int32, self.device),
                                 _dense(top_logit, "top_logit", (n, self.top), torch.float32, self.device),
                                 _dense(teacher_lse, "teacher_lse", (n,), torch.float32, self.device),
                                 fls.FLS_TAIL_RENORM if teacher_lse is None else fls.FLS_TAIL_CLASS, 0, temperature, distill_weight,
                                 label_weight)
        fls.fls_head_distill(self.handle, io, t, self._use(stream))
        return out

    def _io(self, hidden, weight, labels, ignore_label, grad_hidden, grad_weight, row_weight, accumulate, stream):
        dev, dim, io = self.device, self.dim, self._args
        io.hidden, io.hidden_stride = _matrix(hidden, "hidden", None, dim, torch.bfloat16, dev)
        n = hidden.shape[0]
        io.rows = n
        io.weight, io.weight_stride = _matrix(weight, "weight", self.vocab, dim, torch.bfloat16, dev)
        io.labels = _dense(labels, "labels", (n,), torch.int64, dev)
        io.row_weight = _dense(row_weight, "row_weight", (n,), torch.float32, dev)
        io.grad_hidden, io.grad_hidden_stride = (None, 0) if grad_hidden is None else _matrix(grad_hidden, "grad_hidden", n, dim, torch.bfloat16, dev)
        io.grad_weight, io.grad_weight_stride = (None, 0) if grad_weight is None else _matrix(grad_weight, "grad_weight", self.vocab, dim, self.grad_torch_dtype, dev)
        io.ignore_label, io.accumulate = ignore_label, accumulate
        loss, lse = _empty_on(stream, (2, n), torch.float32, dev).unbind(0)
        io.loss, io.lse = loss.data_ptr(), lse.data_ptr()
        return io, (loss, lse)

    def _use(self, stream) -> int:
        """The call's stream as a handle; the workspace's memory is not given to anyone else before its work is done."""
        handle = fls._stream_handle(stream)
        if handle not in self._streams:
            if stream is None:
                stream = torch.cuda.current_stream(self.device)
            elif isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=self.device)
            self.workspace.record_stream(stream)
            self._streams.add(handle)
        return handle

    # ------------------------------------------------------------------ what the device wrote beside the outputs
    def _word(self, i: int) -> torch.Tensor:
        off = fls.fls_head_get_state(self.workspace)[i] - self.workspace.data_ptr()
        return self.workspace[off: off + 4].view(torch.int32)[0]

    def status(self) -> int:
        """FLS_STATUS_* bits of all calls so far (waits for the device)."""
        return int(self._word(0).item())

    def rows_taking_part(self) -> torch.Tensor:
        """Rows of the last call that had a label or a teacher entry: a view on the device, rewritten by the next call."""
        return self._word(1)

    def close(self) -> None:
        if self.handle is not None:
            fls.fls_head_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class TopLogits:
    """A teacher's top logits: for every row of [N, vocab] logits (bf16 or fp32, rows contiguous) the `top` largest in
    descending order, equal ones in ascending index, and the row's log sum exp at `temperature`; the three outputs are what
    `Head.distill` takes as top_logit, top_index and teacher_lse."""

    def __init__(self, max_rows: int, vocab: int, top: int, device: str = "cuda:0"):
        if not torch.cuda.is_available():
            raise RuntimeError("libfls needs a CUDA device; there is no CPU path")
        if not 1 <= top <= fls.FLS_HEAD_MAX_TOP:
            raise ValueError(f"top must be in 1 .. {fls.FLS_HEAD_MAX_TOP}")
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        torch.cuda.set_device(self.device)
        self.max_rows, self.vocab, self.top = max_rows, vocab, top

    def __call__(self, logits: torch.Tensor, temperature: float = 1.0, stream=None):
        """(value fp32 [N, top], index int32 [N, top], lse fp32 [N])"""
        if logits.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"logits must be bf16 or fp32, got {logits.dtype}")
        ptr, stride = _matrix(logits, "logits", None, self.vocab, logits.dtype, self.device)
        n = logits.shape[0]
        if n > self.max_rows:
            raise ValueError(f"{n} rows, made for {self.max_rows}")
        value = _empty_on(stream, (n, self.top), torch.float32, self.device)
        index = _empty_on(stream, (n, self.top), torch.int32, self.device)
        lse = _empty_on(stream, (n,), torch.float32, self.device)
        fls.fls_top_logits(ptr, fls.FLS_GRAD_F32 if logits.dtype == torch.float32 else fls.FLS_GRAD_BF16, n, self.vocab, stride, self.top,
                           temperature, value, index, lse, stream)
        return value, index, lse
