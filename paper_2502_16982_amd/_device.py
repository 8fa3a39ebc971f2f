"""The device and the stream that the operators on torch tensors run on."""
from __future__ import annotations

import contextlib
import warnings

import torch

# the stream's handle without a Stream object around it (a microsecond of every call), where this torch has it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_here = contextlib.nullcontext()


def stream_handle(device: torch.device) -> int:
    """hipStream_t of the current stream of the device."""
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


current_stream = torch.cuda.current_stream
capturing = torch.cuda.is_current_stream_capturing


def outside_autograd(where: str, required: bool) -> None:
    """Warns where an argument requires grad and autograd is on: it does not see these calls, whose gradients are results or calls of their own."""
    if required and torch.is_grad_enabled():
        warnings.warn(f"{where} is not recorded by autograd and an argument requires grad: take the gradients from the results (or from the "
                      f"*_backward calls), and call it under torch.no_grad()", stacklevel=3)


def on(device: torch.device):
    """Context with the device as the current one; nothing to do where it is."""
    return _here if torch.cuda.current_device() == device.index else torch.cuda.device(device)
