"""What the C ABI of the head's losses and of the experts' dispatch refuses before it touches a device (CPU only)."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2502_16982_amd import binding as b
    if not os.path.exists(b.library_path()):
        from paper_2502_16982_amd import build
        build.build_library()
    return b


def head(binding, **over):
    f = dict(hidden=None, weight=None, hidden_stride=64, weight_stride=64, tokens=100, vocab=1000, width=64, dtype=1, reserved=0)
    return binding.muon_head(*{**f, **over}.values())


def test_struct_layouts(binding):
    assert C.sizeof(binding.muon_head) == 7 * 8 + 2 * 4
    assert C.sizeof(binding.muon_routing) == 3 * 8 + 2 * 4


def test_head_workspace(binding):
    size = binding.muon_head_workspace_bytes
    full = size(head(binding), 1, 3)
    assert size(head(binding), 1, 0) < size(head(binding), 1, 1) <= full
    assert full >= 100 * 1024 * 2                                         # the probabilities of all tokens
    assert size(head(binding, tokens=100000), 1, 3) < 2 * size(head(binding, tokens=8192), 1, 3)       # pieces of 8192
    large = head(binding, tokens=8192, vocab=65536, width=1024, hidden_stride=1024, weight_stride=1024)
    assert size(large, 1, 3, 512 << 20) <= 512 << 20 < size(large, 1, 3)   # several pieces: fp32 sums of d_weight, 256 MiB, are part of it
    assert size(large, 1, 1, 64 << 20) <= 64 << 20
    assert size(head(binding, dtype=0), 1, 3) > full
    assert size(head(binding, hidden_stride=67), 1, 3) > full             # rows that are copied first


@pytest.mark.parametrize("over,status", [
    (dict(dtype=2), -2), (dict(dtype=9), -2), (dict(reserved=1), -1), (dict(tokens=-1), -1), (dict(tokens=(1 << 30) + 1), -1),
    (dict(vocab=0), -1), (dict(vocab=(1 << 21) + 1), -1), (dict(width=0), -1), (dict(width=(1 << 20) + 1), -1), (dict(hidden_stride=63), -1),
    (dict(weight_stride=63), -1), (dict(hidden=1), -7), (dict(weight=3), -7), (dict(weight=2, dtype=0), -7)])
def test_head_refusals(binding, over, status):
    L, out = binding.lib(), C.c_size_t(0)
    h = head(binding, **over)
    assert L.muon_head_workspace_bytes(C.byref(h), 1, 3, 0, C.byref(out)) == status
    if over != dict(hidden=1) and over != dict(weight=3) and over != dict(weight=2, dtype=0):
        assert L.muon_cross_entropy(C.byref(h), 8, 8, None, 256, None, None, None, 256, 1 << 40, None) == status
        assert L.muon_distill(C.byref(h), 8, 4, 256, 0, 4, 1.0, None, 256, None, None, None, 256, 1 << 40, None) == status


def test_call_refusals(binding):
    L = binding.lib()
    h = head(binding, hidden=256, weight=256)
    out = C.c_size_t(0)
    assert L.muon_head_workspace_bytes(None, 1, 3, 0, C.byref(out)) == -1
    assert L.muon_head_workspace_bytes(C.byref(h), 1, 3, 0, None) == -1
    for top, gradients in ((0, 3), (4097, 3), (1, 4), (1, -1)):
        assert L.muon_head_workspace_bytes(C.byref(h), top, gradients, 0, C.byref(out)) == -1
    need = binding.muon_head_workspace_bytes(h, 1, 3, 1)

    def ce(h=h, targets=256, size=8, scale=None, loss=256, lse=256, dh=256, dw=256, ws=256, nbytes=need):
        return L.muon_cross_entropy(C.byref(h) if h else None, targets, size, scale, loss, lse, dh, dw, ws, nbytes, None)

    assert ce(h=None) == ce(targets=None) == ce(size=2) == ce(loss=None) == ce(h=head(binding, hidden=256)) == ce(h=head(binding, weight=256)) == -1
    assert ce(targets=4) == ce(targets=2, size=4) == ce(scale=2) == ce(loss=2) == ce(lse=2) == ce(dh=1) == ce(dw=1) == ce(ws=128) == -7
    assert ce(nbytes=need - 256) == ce(nbytes=0) == ce(ws=None) == -4

    def kd(index=256, size=4, logits=256, dtype=0, top=4, tau=1.0):
        return L.muon_distill(C.byref(h), index, size, logits, dtype, top, tau, None, 256, None, None, None, 256, 0, None)

    assert kd(size=3) == kd(logits=None) == kd(top=0) == kd(top=4097) == kd(tau=0.0) == kd(tau=-1.0) == -1
    assert kd(tau=float("inf")) == kd(tau=float("nan")) == kd(tau=1e-50) == kd(tau=1e50) == -1
    assert kd(dtype=2) == -2 and kd(index=2) == kd(logits=2) == -7
    assert kd() == -4


def test_expert_refusals(binding):
    L, out = binding.lib(), C.c_size_t(0)
    assert binding.muon_expert_sort_bytes(100, 6, 64) == 0 and binding.muon_expert_sort_bytes(8192, 6, 64) > 0
    for tokens, top, experts in ((-1, 1, 1), (1, 0, 1), (1, 65, 1), (1, 1, 0), (1, 1, 4097), (1 << 31, 1, 8), (1 << 25, 64, 8)):
        assert L.muon_expert_sort_bytes(tokens, top, experts, C.byref(out)) == -1
        assert L.muon_expert_sort(256, 4, tokens, top, experts, 256, 256, 256, 256, 1 << 40, None) == -1
    assert L.muon_expert_sort_bytes(1, 1, 1, None) == -1

    def sort(expert=256, size=4, tokens=8192, position=256, source=256, offsets=256, ws=256, nbytes=1 << 30):
        return L.muon_expert_sort(expert, size, tokens, 6, 64, position, source, offsets, ws, nbytes, None)

    assert sort(expert=None) == sort(size=8 + 1) == sort(position=None) == sort(source=None) == sort(offsets=None) == -1
    assert sort(expert=2) == sort(expert=4, size=8) == sort(position=1) == sort(source=2) == sort(offsets=3) == sort(ws=2) == -7
    assert sort(ws=None) == sort(nbytes=16) == -4
    r = binding.muon_routing(256, 256, 10, 2, 4)
    for bad, status in ((None, -1), (binding.muon_routing(None, 256, 10, 2, 4), -1), (binding.muon_routing(256, None, 10, 2, 4), -1),
                        (binding.muon_routing(258, 256, 10, 2, 4), -7), (binding.muon_routing(256, 256, 10, 65, 4), -1)):
        assert L.muon_expert_dispatch(C.byref(bad) if bad else None, 256, 16, 16, 1, 256, None) == status
    dispatch = lambda x=256, stride=16, width=16, dtype=1, rows=256: L.muon_expert_dispatch(C.byref(r), x, stride, width, dtype, rows, None)  # noqa: E731
    assert dispatch(x=None) == dispatch(rows=None) == dispatch(stride=15) == dispatch(width=0) == -1
    assert dispatch(dtype=3) == -2 and dispatch(x=1) == dispatch(rows=2, dtype=0) == -7
    combine = lambda rows=256, w=256, out=256, dtype=1: L.muon_expert_combine(C.byref(r), rows, w, 16, dtype, out, None)  # noqa: E731
    assert combine(rows=None) == combine(out=None) == -1 and combine(dtype=7) == -2 and combine(w=2) == combine(out=1) == -7
    back = lambda d=256, s=16, rows=256, w=256, dr=256, dw=256: L.muon_expert_combine_backward(C.byref(r), d, s, rows, w, 16, 1, dr, dw, None)  # noqa: E731
    assert back(d=None) == back(s=3) == back(rows=None) == back(w=None) == back(dr=None) == back(dw=None) == -1
    assert back(d=1) == back(w=1) == back(dw=2) == -7


def test_nothing_to_do_is_not_an_error(binding):
    L = binding.lib()
    r = binding.muon_routing(None, None, 0, 2, 4)
    assert L.muon_expert_dispatch(C.byref(r), None, 16, 16, 1, None, None) == 0
    assert L.muon_expert_combine(C.byref(r), None, None, 16, 1, None, None) == 0
    assert L.muon_expert_combine_backward(C.byref(r), None, 16, None, None, 16, 1, None, None, None) == 0
    h = head(binding, tokens=0, weight=256)
    assert L.muon_cross_entropy(C.byref(h), None, 8, None, None, None, None, None, None, 0, None) == 0
