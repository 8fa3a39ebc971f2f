"""The device and the stream that the operators on torch tensors run on."""
from __future__ import annotations

import contextlib

import torch

# the stream's handle without a Stream object around it (a microsecond of every call), where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_here = contextlib.nullcontext()


def stream_handle(device: torch.device) -> int:
    """hipStream_t of the current stream of the device."""
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


current_stream = torch.cuda.current_stream
capturing = torch.cuda.is_current_stream_capturing


def on(device: torch.device):
    """Context with the device as the current one; nothing to do where it is."""
    return _here if torch.cuda.current_device() == device.index else torch.cuda.device(device)
