"""A mixture's tokens to their experts and back, with gradients.

Argument checks and memory only; the work is in the HIP library (``muon_expert_*``).  Everything runs on the current stream of
the tensors' device.  autograd does not see these calls: ``dispatch_backward`` and ``combine_backward`` are the gradients.
"""
from __future__ import annotations

from functools import lru_cache
from typing import NamedTuple, Optional, Tuple

import torch

from . import binding
from ._device import on, outside_autograd, stream_handle
from .binding import MuonError


class Routing(NamedTuple):
    """position: [tokens, top], the row of each pair or -1; source: [tokens * top], the pair of each row or -1; offsets:
    [experts + 1], first row of each expert and the number of rows.  All int32."""
    position: torch.Tensor
    source: torch.Tensor
    offsets: torch.Tensor


def _device(first: torch.Tensor, *others: Optional[torch.Tensor]) -> torch.device:
    device = first.device
    if device.type != "cuda" or any(t is not None and t.device != device for t in others):
        raise MuonError(-1, f"tensors of one GPU, not {[str(t.device) for t in (first, *others) if t is not None]}")
    return device


def _routing(routing: Routing) -> "binding.muon_routing":
    position, _, offsets = routing
    if position.dim() != 2 or offsets.dim() != 1 or offsets.shape[0] < 2:
        raise MuonError(-1, f"position [tokens, top] and offsets [experts + 1], not {tuple(position.shape)} and {tuple(offsets.shape)}")
    if position.dtype != torch.int32 or offsets.dtype != torch.int32:
        raise MuonError(-2, "position and offsets: int32")
    if not (position.is_contiguous() and offsets.is_contiguous()):
        raise MuonError(-1, "position and offsets must be contiguous")
    return binding.muon_routing(position.data_ptr(), offsets.data_ptr(), position.shape[0], position.shape[1], offsets.shape[0] - 1)


def _tokens(name: str, t: torch.Tensor, tokens: int) -> Tuple[int, int]:
    """(row stride, width) of one row per token."""
    if t.dim() != 2 or t.shape[0] != tokens:
        raise MuonError(-1, f"{name}: [{tokens}, width], not {tuple(t.shape)}")
    if t.stride(1) != 1 and t.shape[1] > 1:
        raise MuonError(-1, f"{name}: rows must be contiguous")
    return (t.stride(0) if tokens > 1 else t.shape[1]), t.shape[1]


def _rows(name: str, t: torch.Tensor, position: torch.Tensor) -> int:
    if t.dim() != 2 or t.shape[0] != position.numel() or not t.is_contiguous():
        raise MuonError(-1, f"{name}: contiguous [{position.numel()}, width], not {tuple(t.shape)}")
    return t.shape[1]


def _weights(t: torch.Tensor, position: torch.Tensor) -> int:
    if t.shape != position.shape or not t.is_contiguous():
        raise MuonError(-1, f"weights: contiguous {tuple(position.shape)}, not {tuple(t.shape)}")
    if t.dtype != torch.float32:
        raise MuonError(-2, f"weights: fp32, not {t.dtype}")
    return t.data_ptr()


_sort_bytes = lru_cache(maxsize=256)(binding.muon_expert_sort_bytes)


def sort_by_expert(expert: torch.Tensor, experts: int) -> Routing:
    """Stable sort of the pairs of ``expert`` [tokens, top] (int32 or int64) by expert; a pair whose expert is not in
    [0, experts) is dropped."""
    if expert.dim() != 2 or not expert.is_contiguous():
        raise MuonError(-1, f"expert: contiguous [tokens, top], not {tuple(expert.shape)}")
    if expert.dtype not in (torch.int32, torch.int64):
        raise MuonError(-2, f"expert: int32 or int64, not {expert.dtype}")
    device = _device(expert)
    tokens, top = expert.shape
    need = _sort_bytes(tokens, top, experts)
    with on(device):
        # one allocation for what is written; the workspace goes back to the stream it was used on
        pairs = tokens * top
        ints = torch.empty(2 * pairs + experts + 1, dtype=torch.int32, device=device)
        position, source, offsets = ints[:pairs].view(tokens, top), ints[pairs:2 * pairs], ints[2 * pairs:]
        workspace = torch.empty(need, dtype=torch.uint8, device=device) if need else None
        binding.muon_expert_sort(expert.data_ptr(), expert.element_size(), tokens, top, experts, position.data_ptr(), source.data_ptr(),
                                 offsets.data_ptr(), 0 if workspace is None else workspace.data_ptr(), need, stream_handle(device))
    return Routing(position, source, offsets)


def dispatch(x: torch.Tensor, routing: Routing) -> torch.Tensor:
    """Rows [tokens * top, width] of ``x`` [tokens, width] in the experts' order; zero behind the last pair's."""
    r, device = _routing(routing), _device(x, routing.position, routing.offsets)
    stride, width = _tokens("x", x, r.tokens)
    outside_autograd("experts.dispatch", x.requires_grad)
    with on(device):
        rows = torch.empty(r.tokens * r.top, width, dtype=x.dtype, device=device)
        binding.muon_expert_dispatch(r, x.data_ptr(), stride, width, binding.dtype_code(x.dtype), rows.data_ptr(), stream_handle(device))
    return rows


def dispatch_backward(d_rows: torch.Tensor, routing: Routing) -> torch.Tensor:
    """Gradient [tokens, width] of what ``dispatch`` took."""
    return combine(d_rows, None, routing)


def combine(rows: torch.Tensor, weights: Optional[torch.Tensor], routing: Routing) -> torch.Tensor:
    """[tokens, width]: the sum of each token's rows, times ``weights`` [tokens, top] in fp32 (None: all 1)."""
    r = _routing(routing)
    device = _device(rows, weights, routing.position, routing.offsets)
    width, at = _rows("rows", rows, routing.position), 0 if weights is None else _weights(weights, routing.position)
    outside_autograd("experts.combine", rows.requires_grad or (weights is not None and weights.requires_grad))
    with on(device):
        out = torch.empty(r.tokens, width, dtype=rows.dtype, device=device)
        binding.muon_expert_combine(r, rows.data_ptr(), at, width, binding.dtype_code(rows.dtype), out.data_ptr(), stream_handle(device))
    return out


def combine_backward(d_out: torch.Tensor, rows: torch.Tensor, weights: torch.Tensor, routing: Routing) -> Tuple[torch.Tensor, torch.Tensor]:
    """(d_rows, d_weights) of ``combine(rows, weights, routing)`` for its result's gradient."""
    r = _routing(routing)
    device = _device(d_out, rows, weights, routing.position, routing.offsets)
    width, at = _rows("rows", rows, routing.position), _weights(weights, routing.position)
    stride, d_width = _tokens("d_out", d_out, r.tokens)
    if d_width != width:
        raise MuonError(-1, f"d_out: [{r.tokens}, {width}], not {tuple(d_out.shape)}")
    if d_out.dtype != rows.dtype:
        raise MuonError(-2, f"d_out and rows of one dtype, not {d_out.dtype} and {rows.dtype}")
    outside_autograd("experts.combine_backward", d_out.requires_grad or rows.requires_grad or weights.requires_grad)
    with on(device):
        d_rows, d_weights = torch.empty_like(rows), torch.empty_like(weights)
        binding.muon_expert_combine_backward(r, d_out.data_ptr(), stride, rows.data_ptr(), at, width, binding.dtype_code(rows.dtype),
                                             d_rows.data_ptr(), d_weights.data_ptr(), stream_handle(device))
    return d_rows, d_weights
