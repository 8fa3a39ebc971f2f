"""The norm of all gradients of a step, and clipping by it.

Argument checks and memory only; the arithmetic is in the HIP library (``muon_grad_*``).  Everything runs on the current stream of
the gradients' device.
"""
from __future__ import annotations

import math
from typing import Iterable, NamedTuple

import torch

from . import binding
from ._device import on, stream_handle
from .binding import MuonError


class ClipScale(NamedTuple):
    """norm: one fp64 element, the norm of the gradients as they came; scale: one fp32 element, what they count times."""
    norm: torch.Tensor
    scale: torch.Tensor


class GradClipper:
    """The gradients of one step: contiguous fp32 or bf16 tensors of any shape on one GPU.

    Their addresses are read here and by ``set_grads``, not at every call.  Calls may come on any stream and be captured; what they need
    is allocated with them.
    """

    def __init__(self, grads: Iterable[torch.Tensor]):
        self.set_grads(grads)

    def set_grads(self, grads: Iterable[torch.Tensor]) -> None:
        grads = list(grads)
        if not grads:
            raise MuonError(-1, "empty list of gradients")
        device = grads[0].device
        array = (binding.muon_grad * len(grads))()
        for i, g in enumerate(grads):
            if g.device != device or (g.device.type != "cuda" and g.device != torch.device("cpu")):
                raise MuonError(-1, f"gradient {i} is on {g.device}, the first one on {device}")
            if not g.is_contiguous():
                raise MuonError(-1, f"gradient {i} must be contiguous")
            array[i].g, array[i].numel, array[i].dtype = g.data_ptr(), g.numel(), binding.dtype_code(g.dtype)
        need = binding.muon_grad_norm_bytes(array, len(grads))
        self.grads, self.device, self._array, self._need = grads, device, array, need

    def _on_gpu(self) -> None:
        if self.device.type != "cuda":
            raise MuonError(-1, f"gradients on a GPU, not on {self.device}")

    def _call(self, entry, max_norm: float) -> ClipScale:
        self._on_gpu()
        with on(self.device):
            norm = torch.empty((), dtype=torch.float64, device=self.device)
            scale = torch.empty((), dtype=torch.float32, device=self.device)
            workspace = torch.empty(self._need, dtype=torch.uint8, device=self.device)
            entry(self._array, len(self.grads), max_norm, norm.data_ptr(), scale.data_ptr(), workspace.data_ptr(), self._need,
                  stream_handle(self.device))
        return ClipScale(norm, scale)

    def scale(self, max_norm: float = math.inf) -> ClipScale:
        """Norm, and the scale that brings it down to ``max_norm`` (1 where it is not above, or not finite).  The gradients are read only: give
        ``scale`` to ``MuonStepper.step`` and ``muon_adamw_step`` as ``grad_scale``."""
        return self._call(binding.muon_grad_norm, max_norm)

    def clip_(self, max_norm: float) -> ClipScale:
        """The same, and the gradients scaled in place (not touched where the scale is 1)."""
        return self._call(binding.muon_grad_clip, max_norm)

    def scale_(self, scale: torch.Tensor) -> None:
        """The gradients times one fp32 element on their device, such as a scale from the norm over several processes, in place."""
        self._on_gpu()
        with on(self.device):
            binding.muon_grad_scale(self._array, len(self.grads), binding.grad_scale_ptr(scale, self.device), stream_handle(self.device))
