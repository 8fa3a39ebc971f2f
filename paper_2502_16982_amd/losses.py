"""Losses of a language model's head with their gradients: softmax cross entropy over a large vocabulary and distillation
from a teacher's top logits, from hidden states and the head's weight, without keeping the logits; and log probabilities of given tokens
with entropies and top alternatives, from the same, with a backward call of their own, for which the first one may keep the logits' powers.

Argument checks and memory only; the arithmetic is in the HIP library (``muon_cross_entropy``, ``muon_distill``, ``muon_log_probs``).
autograd does not see these calls: the losses' gradients are in their results, for the token_scale given.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import binding
from ._device import capturing, current_stream, on, outside_autograd, stream_handle
from .binding import MuonError


# What ``log_probs`` keeps unasked for at most: what 32768 tokens of a vocabulary of 131072 take in bf16, a thirty-sixth of the card's memory.
KEEP_BYTES = 8 << 30


class HeadResult(NamedTuple):
    """loss and lse: [tokens] in fp32; d_hidden, d_weight: in the inputs' type, or None where not asked for."""
    loss: torch.Tensor
    lse: torch.Tensor
    d_hidden: Optional[torch.Tensor]
    d_weight: Optional[torch.Tensor]


class TokenScores(NamedTuple):
    """log_prob: [tokens] in fp32, or None without targets; entropy, lse: [tokens] in fp32; lse_rest: what fp32 leaves of lse; top_index:
    [tokens, top] in int64, top_log_prob: in fp32, or None where not asked for; kept: what ``log_probs_backward`` reads instead of making the logits
    once more, or None."""
    log_prob: Optional[torch.Tensor]
    entropy: torch.Tensor
    lse: torch.Tensor
    lse_rest: torch.Tensor
    top_index: Optional[torch.Tensor]
    top_log_prob: Optional[torch.Tensor]
    kept: Optional[torch.Tensor] = None


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
        self.gradients = bool(gradients)
        self.workspace = None
        self._stream = None                                # handle and object of the stream that used the workspace last
        self._last = None
        self._captured = False                             # whether a graph holds the workspace's address
        self._kept = []                                    # replaced workspaces of which that is so
        self._sizes = {}
        head = binding.muon_head(None, None, width, width, tokens, vocab, width, binding.dtype_code(dtype), 0)
        self._fit(head, top, 3 if gradients else 0)

    def _fit(self, head: "binding.muon_head", top: int, gradients: int, scores: bool = False) -> int:
        """Bytes of workspace for the call (scores: of ``log_probs``), which are there then.  The library cuts the call by these and not by all
        that there is, so that results do not depend on earlier calls."""
        # what the size goes by: the pointers for their alignment only
        key = (head.tokens, head.vocab, head.width, head.hidden_stride, head.weight_stride, head.dtype, (head.hidden or 0) % 16,
               (head.weight or 0) % 16, top, gradients, scores)
        need = self._sizes.get(key)
        if need is None:
            need = (binding.muon_log_probs_bytes(head, top, self.max_workspace_bytes) if scores else
                    binding.muon_head_workspace_bytes(head, top, gradients, self.max_workspace_bytes))
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

    def _gradients(self, hidden, weight, gradients):
        """gradients: True, False, or the names of those wanted."""
        wanted = {True: ("hidden", "weight"), False: ()}.get(gradients, gradients) if isinstance(gradients, bool) else tuple(gradients)
        if not set(wanted) <= {"hidden", "weight"}:
            raise ValueError("gradients: True, False, or a sequence of 'hidden' and 'weight'")
        dh = torch.empty(hidden.shape, dtype=hidden.dtype, device=self.device) if "hidden" in wanted else None
        dw = torch.empty(weight.shape, dtype=weight.dtype, device=self.device) if "weight" in wanted else None
        return dh, dw

    def _outputs(self, hidden, weight, gradients):
        dh, dw = self._gradients(hidden, weight, gradients)
        loss, lse = torch.empty(2, hidden.shape[0], dtype=torch.float32, device=self.device).unbind(0)
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

    def _targets(self, targets: Optional[torch.Tensor], tokens: int):
        """(address, bytes of an index); no targets: (0, 8)."""
        if targets is None:
            return 0, 8
        if targets.shape != (tokens,) or not targets.is_contiguous():
            raise MuonError(-1, f"targets: contiguous [{tokens}], not {tuple(targets.shape)}")
        return targets.data_ptr(), _index_bytes(targets, "targets")

    def log_probs(self, hidden: torch.Tensor, weight: torch.Tensor, targets: Optional[torch.Tensor] = None, top: int = 0,
                  temperature: float = 1.0, keep: Optional[bool] = None) -> TokenScores:
        """Log probabilities of ``targets`` (negative: no token, 0) under the softmax of ``hidden @ weight.T / temperature``, the entropy of
        each row's whole distribution, and its ``top`` (up to 64) most likely entries with their log probabilities, the likeliest first, equal
        ones by index.  keep: whether the result holds what ``log_probs_backward`` saves one of its three products by, 2 bytes per token and vocabulary
        entry (fp32: 4) beside the workspace, as long as the result lives; only without alternatives, and not for few tokens where it saves nothing;
        None: where the LossHead is for gradients and that is no more than its max_workspace_bytes or, without such a limit, 8 GiB."""
        head = self._head(hidden, weight)
        self._here(hidden=hidden, weight=weight, targets=targets)
        outside_autograd("LossHead.log_probs", hidden.requires_grad or weight.requires_grad)
        tokens = hidden.shape[0]
        at, size = self._targets(targets, tokens)
        with on(self.device):
            need = self._fit(head, top, 0, scores=True)
            kept, kept_bytes = None, 0
            if keep or (keep is None and self.gradients and not top):
                kept_bytes = binding.muon_log_probs_kept_bytes(head)
                if kept_bytes and (keep or kept_bytes <= (self.max_workspace_bytes or KEEP_BYTES)):
                    kept = torch.empty(kept_bytes, dtype=torch.uint8, device=self.device)
            values = torch.empty(4, tokens, dtype=torch.float32, device=self.device).unbind(0)
            out = TokenScores(None if targets is None else values[0], *values[1:],
                              torch.empty(tokens, top, dtype=torch.int64, device=self.device) if top else None,
                              torch.empty(tokens, top, dtype=torch.float32, device=self.device) if top else None, kept)
            binding.muon_log_probs(head, at, size, top, temperature, *(0 if t is None else t.data_ptr() for t in out), kept_bytes,
                                   self.workspace.data_ptr(), need, stream_handle(self.device))
        return out

    def log_probs_backward(self, hidden: torch.Tensor, weight: torch.Tensor, targets: Optional[torch.Tensor], scores: TokenScores,
                           d_log_prob: Optional[torch.Tensor], d_entropy: Optional[torch.Tensor] = None, temperature: float = 1.0,
                           gradients=True) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
        """(d_hidden, d_weight) of ``(d_log_prob * log_prob + d_entropy * entropy).sum()`` with the ``scores`` that ``log_probs`` gave for the
        same hidden states, weight, targets and temperature.  ``d_log_prob`` is None without targets, ``d_entropy`` None for 0."""
        head = self._head(hidden, weight)
        self._here(hidden=hidden, weight=weight, targets=targets, d_log_prob=d_log_prob, d_entropy=d_entropy, lse=scores.lse, lse_rest=scores.lse_rest,
                   entropy=scores.entropy, kept=scores.kept)
        outside_autograd("LossHead.log_probs_backward", hidden.requires_grad or weight.requires_grad)
        tokens = hidden.shape[0]
        at, size = self._targets(targets, tokens)
        if (targets is None) != (d_log_prob is None):
            raise MuonError(-1, "targets and d_log_prob: both or neither")
        if d_log_prob is None and d_entropy is None:
            raise MuonError(-1, "d_log_prob or d_entropy")
        kept = scores.kept
        if kept is not None and kept.numel() != (binding.muon_log_probs_kept_bytes(head) or kept.numel()):
            raise MuonError(-1, "scores.kept: of another call's sizes")         # (0: a call whose own rows would be copied; it makes the logits again)
        given = []
        for name, t in (("lse", scores.lse), ("lse_rest", scores.lse_rest), ("entropy", scores.entropy), ("d_log_prob", d_log_prob),
                        ("d_entropy", d_entropy)):
            if t is not None and (t.shape != (tokens,) or not t.is_contiguous()):
                raise MuonError(-1, f"{name}: contiguous [{tokens}], not {tuple(t.shape)}")
            if t is not None and t.dtype != torch.float32:
                raise MuonError(-2, f"{name}: fp32, not {t.dtype}")
            given.append(0 if t is None else t.data_ptr())
        with on(self.device):
            dh, dw = self._gradients(hidden, weight, gradients)
            need = self._fit(head, 1, (1 if dh is not None else 0) | (2 if dw is not None else 0))
            binding.muon_log_probs_backward(head, at, size, temperature, *given, 0 if kept is None else kept.data_ptr(),
                                            0 if kept is None else kept.numel(), *(0 if t is None else t.data_ptr() for t in (dh, dw)),
                                            self.workspace.data_ptr(), need, stream_handle(self.device))
        return dh, dw
