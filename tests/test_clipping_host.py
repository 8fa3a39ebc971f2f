"""The gradients' norm and clipping without a GPU: refusals of the C ABI and of the binding, and the cutting of lists into launches."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

from paper_2502_16982_amd import binding, clipping

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20                                             # an address that nothing reads before it is refused


def array(*grads):
    """grads: (address, numel, dtype)"""
    out = (binding.muon_grad * max(1, len(grads)))()
    for o, (g, n, d) in zip(out, grads):
        o.g, o.numel, o.dtype = g, n, d
    return out, len(grads)


def test_workspace_grows_with_the_list():
    sizes = [binding.muon_grad_norm_bytes(*array(*[(0, n, 1)] * k)) for n, k in ((0, 0), (1, 1), (16384, 4), (16385, 40), (1 << 34, 1), (1 << 42, 3))]
    assert sizes == sorted(sizes) and sizes[0] >= 8 and sizes[-1] >= 3 * (1 << 42) // 16384 * 8


def test_refusals():
    L = binding.lib()
    need, out = 1 << 12, C.c_size_t(0)
    ok, n = array((FAKE, 100, 1), (FAKE + 4096, 50, 0))
    assert L.muon_grad_norm_bytes(ok, n, None) == -1
    assert L.muon_grad_norm_bytes(None, 1, C.byref(out)) == -1
    assert L.muon_grad_norm_bytes(ok, -1, C.byref(out)) == -1
    for bad, status in ((array((FAKE, -1, 1)), -1), (array((FAKE, (1 << 42) + 1, 1)), -1), (array((FAKE, 4, 2)), -2), (array((0, 4, 1)), -1),
                        (array((FAKE + 1, 4, 1)), -7), (array((FAKE + 2, 4, 0)), -7)):
        assert L.muon_grad_norm(*bad, 1.0, FAKE, FAKE, FAKE, need, None) == status
        assert L.muon_grad_clip(*bad, 1.0, FAKE, FAKE, FAKE, need, None) == status
        assert L.muon_grad_scale(*bad, FAKE, None) == status
    reserved, n1 = array((FAKE, 4, 1))
    reserved[0].reserved = 1
    assert L.muon_grad_norm(reserved, n1, 1.0, FAKE, FAKE, FAKE, need, None) == -1
    for entry in (L.muon_grad_norm, L.muon_grad_clip):
        assert entry(ok, n, -1.0, FAKE, FAKE, FAKE, need, None) == -1
        assert entry(ok, n, math.nan, FAKE, FAKE, FAKE, need, None) == -1
        assert entry(ok, n, 1.0, None, FAKE, FAKE, need, None) == -1
        assert entry(ok, n, 1.0, FAKE, FAKE, None, need, None) == -4
        assert entry(ok, n, 1.0, FAKE, FAKE, FAKE, 8, None) == -4
        assert entry(ok, n, 1.0, FAKE + 4, FAKE, FAKE, need, None) == -7
        assert entry(ok, n, 1.0, FAKE, FAKE + 2, FAKE, need, None) == -7
        assert entry(ok, n, 1.0, FAKE, FAKE, FAKE + 4, need, None) == -7
    assert L.muon_grad_clip(ok, n, 1.0, FAKE, None, FAKE, need, None) == -1
    assert L.muon_grad_scale(ok, n, None, None) == -1
    assert L.muon_grad_scale(ok, n, FAKE + 2, None) == -7


@pytest.mark.parametrize("grads", [((FAKE, 100, 1), (FAKE, 100, 1)), ((FAKE, 100, 1), (FAKE + 198, 4, 1)), ((FAKE + 396, 1, 0), (FAKE, 100, 0)),
                                   ((FAKE + 4096, 8, 1), (FAKE, 8, 0), (FAKE + 28, 8, 1))])
def test_tensors_that_share_memory_are_not_scaled(grads):
    L = binding.lib()
    assert L.muon_grad_scale(*array(*grads), FAKE, None) == -1
    assert L.muon_grad_clip(*array(*grads), 1.0, FAKE, FAKE, FAKE, 1 << 12, None) == -1


def test_binding_refuses():
    with pytest.raises(binding.MuonError):
        clipping.GradClipper([])
    with pytest.raises(binding.MuonError):
        clipping.GradClipper([torch.zeros(4, 4).T[1:]])
    with pytest.raises(binding.MuonError):
        clipping.GradClipper([torch.zeros(4, dtype=torch.float16)])
    on_cpu = clipping.GradClipper([torch.zeros(4), torch.zeros(0)])
    for call in (on_cpu.scale, on_cpu.clip_):
        with pytest.raises(binding.MuonError):
            call(1.0)
    with pytest.raises(binding.MuonError):
        binding.grad_scale_ptr(torch.ones(2), torch.device("cpu"))
    with pytest.raises(binding.MuonError):
        binding.grad_scale_ptr(torch.ones(1, dtype=torch.float64), torch.device("cpu"))
    with pytest.raises(binding.MuonError):
        binding.grad_scale_ptr(torch.ones(1), torch.device("cuda:0"))
    assert binding.lib().muon_step_scaled(None, None, 0, None, 2, None, None) == -7
    assert binding.lib().muon_adamw_step_scaled(None, 0, None, 2, None) == -7


def test_lists_are_cut_into_whole_spans(tmp_path):
    """Every element once, in its tensor's order, whatever the sizes; more tensors than slots, tensors beyond a launch."""
    exe = str(tmp_path / "clip_batch")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "clip_batch_main.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr
    assert "ok" in out.stdout


def test_scaling_refuses_gradients_that_are_not_on_a_gpu():
    on_cpu = clipping.GradClipper([torch.zeros(4), torch.zeros(0)])
    with pytest.raises(binding.MuonError, match="on a GPU"):
        on_cpu.scale_(torch.ones(1))
