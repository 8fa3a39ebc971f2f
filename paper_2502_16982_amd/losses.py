"""Losses of a language model's head with their gradients: softmax cross entropy over a large vocabulary and distillation
from a teacher's top logits, from hidden states and the head's weight, without keeping the logits.

Argument checks and memory only; the arithmetic is in the HIP library (``muon_cross_entropy``, ``muon_distill``).  autograd does not see
these calls: the gradients are in their results, for the token_scale given.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding
from ._device import capturing, current_stream, on, outside_autograd, stream_handle
from .binding import MuonError


class HeadResult(NamedTuple):
    """loss and lse: [tokens] in fp32; d_hidden, d_weight: in the inputs' type, or None where not asked for."""
    loss: torch.Tensor
    lse: torch.Tensor
    d_hidden: Optional[torch.Tensor]
    d_weight: Optional[torch.Tensor]


def _index_bytes(t: torch.Tensor, what: str) -> int:
    if t.dtype not in (torch.int32, torch.int64):
        raise MuonError(-2, f"{what}: int32 or int64, not {t.dtype}")
    return t.element_size()


class LossHead:
    """Workspace of a head's losses and the calls that use it.

    tokens, vocab, width, dtype, top (entries per token of ``distill``): the largest call to expect; smaller ones use the same
    workspace, a larger one replaces it, and so does one whose rows are copied first (bf16 of a width, stride or address that is no
    multiple of 16 bytes, where the declared width is one).  max_workspace_bytes: limit of the workspace, in exchange for smaller
    pieces of tokens (0: what pieces of 8192 tokens take).  gradients: whether calls will ask for any (they may all the same).  Calls run
    on the current stream of the device, on another one than the call before behind that call: streams that are to run at a time
    need a LossHead each, and so do host threads.  Captured calls are ordered by their capture alone and keep the workspace that they
    were captured with as long as the LossHead is there: keep it while their graphs are replayed, and replay none beside other calls
    of it.
    """

    def __init__(self, tokens: int, vocab: int, width: int, dtype: torch.dtype = torch.bfloat16, max_workspace_bytes: int = 0,
                 gradients: bool = True, device="cuda", top: int = 64):
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.max_workspace_bytes = int(max_workspace_bytes)
        self.dtype = dtype
        self.workspace = None
        self._stream = None                                # handle and object of the stream that used the workspace last
        self._last = None
        self._captured = False                             # whether a graph holds the workspace's address
        self._kept = []                                    # replaced workspaces of which that is so
        self._sizes = {}
        head = binding.muon_head(None, None, width, width, tokens, vocab, width, binding.dtype_code(dtype), 0)
        self._fit(head, top, 3 if gradients else 0)

    def _fit(self, head: "binding.muon_head", top: int, gradients: int) -> int:
        """Bytes of workspace for the call, which are there then.  The library cuts the call by these and not by all that there is, so that
        results do not depend on earlier calls."""
        # what the size goes by: the pointers for their alignment only
        key = (head.tokens, head.vocab, head.width, head.hidden_stride, head.weight_stride, head.dtype, (head.hidden or 0) % 16,
               (head.weight or 0) % 16, top, gradients)
        need = self._sizes.get(key)
        if need is None:
            need = binding.muon_head_workspace_bytes(head, top, gradients, self.max_workspace_bytes)
            if len(self._sizes) > 1000:
                self._sizes.clear()
            self._sizes[key] = need
        stream = stream_handle(self.device)
        if self.workspace is None or self.workspace.numel() < need:
            if self._captured:
                self._kept.append(self.workspace)
                self._captured = False
            self.workspace = None                          # its memory may serve the next one
            self.workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            self._stream, self._last = stream, current_stream(self.device)
        elif stream != self._stream:                       # after the last call; and the memory outlives what this stream does with it
            now = current_stream(self.device)
            if not capturing():
                now.wait_stream(self._last)
            self.workspace.record_stream(now)
            self._stream, self._last = stream, now
        self._captured = self._captured or capturing()
        return need

    def _head(self, hidden: torch.Tensor, weight: torch.Tensor) -> "binding.muon_head":
        if hidden.dim() != 2 or weight.dim() != 2 or hidden.shape[1] != weight.shape[1]:
            raise MuonError(-1, f"hidden [tokens, width] and weight [vocab, width], not {tuple(hidden.shape)} and {tuple(weight.shape)}")
        if hidden.dtype != weight.dtype:
            raise MuonError(-2, f"hidden and weight of one dtype, not {hidden.dtype} and {weight.dtype}")
        for name, t in (("hidden", hidden), ("weight", weight)):
            if t.stride(1) != 1 and t.shape[1] > 1:
                raise MuonError(-1, f"{name}: rows must be contiguous")
        tokens, width = hidden.shape
        strides = [t.stride(0) if t.shape[0] > 1 else width for t in (hidden, weight)]
        return binding.muon_head(hidden.data_ptr(), weight.data_ptr(), *strides, tokens, weight.shape[0], width,
                                 binding.dtype_code(hidden.dtype), 0)

    def _here(self, **tensors) -> None:
        for name, t in tensors.items():
            if t is not None and t.device != self.device:
                raise MuonError(-1, f"{name} is on {t.device}, the workspace on {self.device}")

    def _scale(self, token_scale, tokens: int) -> int:
        if token_scale is None:
            return 0
        if token_scale.dtype != torch.float32:
            raise MuonError(-2, f"token_scale: fp32, not {token_scale.dtype}")
        if token_scale.shape != (tokens,) or not token_scale.is_contiguous():
            raise MuonError(-1, f"token_scale: contiguous [{tokens}], not {tuple(token_scale.shape)}")
        return token_scale.data_ptr()

    def _outputs(self, hidden, weight, gradients):
        """gradients: True, False, or the names of those wanted."""
        wanted = {True: ("hidden", "weight"), False: ()}.get(gradients, gradients) if isinstance(gradients, bool) else tuple(gradients)
        if not set(wanted) <= {"hidden", "weight"}:
            raise ValueError("gradients: True, False, or a sequence of 'hidden' and 'weight'")
        tokens = hidden.shape[0]
        loss, lse = torch.empty(2, tokens, dtype=torch.float32, device=self.device).unbind(0)
        dh = torch.empty(hidden.shape, dtype=hidden.dtype, device=self.device) if "hidden" in wanted else None
        dw = torch.empty(weight.shape, dtype=weight.dtype, device=self.device) if "weight" in wanted else None
        return HeadResult(loss, lse, dh, dw), (1 if dh is not None else 0) | (2 if dw is not None else 0)

    @staticmethod
    def _pointers(r: HeadResult):
        return r.loss.data_ptr(), r.lse.data_ptr(), *(0 if t is None else t.data_ptr() for t in (r.d_hidden, r.d_weight))

    def cross_entropy(self, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                      token_scale: Optional[torch.Tensor] = None, gradients=True) -> HeadResult:
        """Softmax cross entropy of ``hidden @ weight.T`` against ``targets`` (negative: ignored).  The gradients are those of
        ``(token_scale * loss).sum()``."""
        head = self._head(hidden, weight)
        self._here(hidden=hidden, weight=weight, targets=targets, token_scale=token_scale)
        outside_autograd("LossHead.cross_entropy", hidden.requires_grad or weight.requires_grad)
        if targets.shape != (hidden.shape[0],) or not targets.is_contiguous():
            raise MuonError(-1, f"targets: contiguous [{hidden.shape[0]}], not {tuple(targets.shape)}")
        size, scale = _index_bytes(targets, "targets"), self._scale(token_scale, hidden.shape[0])
        with on(self.device):
            out, which = self._outputs(hidden, weight, gradients)
            need = self._fit(head, 1, which)
            binding.muon_cross_entropy(head, targets.data_ptr(), size, scale, *self._pointers(out), self.workspace.data_ptr(), need,
                                       stream_handle(self.device))
        return out

    def distill(self, hidden: torch.Tensor, weight: torch.Tensor, teacher_index: torch.Tensor, teacher_logits: torch.Tensor,
                temperature: float = 1.0, token_scale: Optional[torch.Tensor] = None, gradients=True) -> HeadResult:
        """``temperature**2`` times the divergence of the softmax of ``hidden @ weight.T / temperature`` from the softmax of the
        teacher's logits (over the temperature) on its ``teacher_index`` (negative: no entry).  The gradients are those of
        ``(token_scale * loss).sum()``."""
        head = self._head(hidden, weight)
        self._here(hidden=hidden, weight=weight, teacher_index=teacher_index, teacher_logits=teacher_logits, token_scale=token_scale)
        outside_autograd("LossHead.distill", hidden.requires_grad or weight.requires_grad or teacher_logits.requires_grad)
        if teacher_index.dim() != 2 or teacher_index.shape[0] != hidden.shape[0] or teacher_logits.shape != teacher_index.shape:
            raise MuonError(-1, f"teacher_index and teacher_logits: [{hidden.shape[0]}, top], not {tuple(teacher_index.shape)} and "
                                f"{tuple(teacher_logits.shape)}")
        if not (teacher_index.is_contiguous() and teacher_logits.is_contiguous()):
            raise MuonError(-1, "teacher_index and teacher_logits must be contiguous")
        size, scale, top = _index_bytes(teacher_index, "teacher_index"), self._scale(token_scale, hidden.shape[0]), teacher_index.shape[1]
        with on(self.device):
            out, which = self._outputs(hidden, weight, gradients)
            need = self._fit(head, top, which)
            binding.muon_distill(head, teacher_index.data_ptr(), size, teacher_logits.data_ptr(), binding.dtype_code(teacher_logits.dtype),
                                 top, temperature, scale, *self._pointers(out), self.workspace.data_ptr(), need,
                                 stream_handle(self.device))
        return out
