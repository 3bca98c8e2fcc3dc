"""What the calls of an operator share: device memory, one call at a time, and argument structures, one set per host thread."""
from __future__ import annotations

import ctypes
import threading

import torch

from . import _binding as fls

_current_raw_stream = torch._C._cuda_getCurrentRawStream


def device_of(device) -> torch.device:
    """The CUDA device, made current."""
    if not torch.cuda.is_available():
        raise RuntimeError("libfls needs a CUDA device; there is no CPU path")
    device = torch.device(device)
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    torch.cuda.set_device(device)
    return device


def dtype_of(name: str, what: str):
    """(torch's type, the library's) of "bf16" or "f32"."""
    if name not in ("bf16", "f32"):
        raise ValueError(f"{what} must be 'bf16' or 'f32'")
    return (torch.float32, fls.FLS_GRAD_F32) if name == "f32" else (torch.bfloat16, fls.FLS_GRAD_BF16)


def matrix(t: torch.Tensor, name: str, rows, cols: int, dtype: torch.dtype):
    """Checks a 2-D tensor whose rows are contiguous and do not overlap; returns (address, elements between rows, 0 if dense)."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 2 or shape[1] != cols or (rows is not None and shape[0] != rows) or not t.is_cuda:
        raise ValueError(f"{name} must be a {dtype} tensor of shape [{'N' if rows is None else rows}, {cols}] on a CUDA device, "
                         f"got {t.dtype} {tuple(shape)} on {t.device}")
    if t.is_contiguous():                                  # another device than the current one is the library's to refuse
        return t.data_ptr(), 0
    row, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous (stride {one})")
    if row < cols:
        raise ValueError(f"{name}: rows overlap (stride {row})")
    return t.data_ptr(), row


def vector(t, name: str, n: int, dtype: torch.dtype):
    """Address of a contiguous tensor of n elements, None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.dim() != 1 or t.numel() != n or not t.is_contiguous() or not t.is_cuda:
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {(n,)} on a CUDA device, got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


class Arguments(threading.local):
    """Argument structures of the calls in preparation, as (type, fields that stay) by name; `name`_ref is what the library takes.
    Each host thread has its own: the interpreter may switch threads between two fields, and does while the library reads them."""

    def __init__(self, **kinds):
        for name, (kind, fields) in kinds.items():
            io = kind(**fields)
            setattr(self, name, io)
            setattr(self, name + "_ref", ctypes.byref(io))


class Workspace:
    """`nbytes` of memory, the first 256 of them zero, that nothing else uses from here on, whichever stream the first call is on, and that is not given to
    anyone else before the work of every call is done; and the streams and outputs of those calls."""

    def __init__(self, nbytes: int, device: torch.device):
        self.device = device
        self.memory = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.memory[:256].zero_()
        # the clear, and what used this memory before, must not come after the first call
        self._clear = not torch.cuda.is_current_stream_capturing()
        if self._clear:
            torch.cuda.current_stream(device).synchronize()
        # otherwise only the graph's replays clear it, and a call that is not in that graph may come before the first of them
        self._streams = {fls._stream_handle(None)}             # those that torch's allocator knows to use the memory
        self._like = {t: torch.empty(0, dtype=t, device=device) for t in (torch.float32, torch.bfloat16)}

    def stream(self, stream) -> int:
        """The call's stream as a handle."""
        return _current_raw_stream(self.device.index) if stream is None else fls._stream_handle(stream)

    def use(self, stream) -> int:
        """The same, for a call that uses the memory."""
        handle = self.stream(stream)
        if handle not in self._streams:
            self.memory.record_stream(self._torch_stream(stream))
            self._streams.add(handle)
        if not self._clear:
            with torch.cuda.stream(self._torch_stream(stream)):
                self.memory[:256].zero_()
                self._clear = not torch.cuda.is_current_stream_capturing()
        return handle

    def new(self, stream, shape, dtype: torch.dtype) -> torch.Tensor:
        """An output of a call: its memory's reuse is ordered by the stream that writes it, which need not be torch's current one."""
        if stream is None:
            return self._like[dtype].new_empty(shape)
        with torch.cuda.stream(self._torch_stream(stream)):
            return torch.empty(shape, dtype=dtype, device=self.device)

    def _torch_stream(self, stream):
        if stream is None:
            return torch.cuda.current_stream(self.device)
        return torch.cuda.ExternalStream(stream, device=self.device) if isinstance(stream, int) else stream
