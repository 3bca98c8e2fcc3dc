"""Device memory that an operator's calls share, one call at a time."""
from __future__ import annotations

import torch

from . import _binding as fls


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


class Workspace:
    """`nbytes` of memory that nothing else uses from here on, whichever stream the first call is on; it is not given to
    anyone else before the work of every call is done."""

    def __init__(self, nbytes: int, device: torch.device):
        self.device = device
        self.memory = torch.empty(nbytes, dtype=torch.uint8, device=device)
        # what used this memory before must not come after the first call
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream(device).synchronize()
        self._streams = {fls._stream_handle(None)}             # those that torch's allocator knows to use the memory

    def use(self, stream) -> int:
        """The call's stream as a handle."""
        handle = fls._stream_handle(stream)
        if handle not in self._streams:
            if stream is None:
                stream = torch.cuda.current_stream(self.device)
            elif isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=self.device)
            self.memory.record_stream(stream)
            self._streams.add(handle)
        return handle
