"""A mixture's layer for few tokens without a GPU: refusals of the C ABI and of the binding, how a call is cut up, the oracle's own pins."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import layer_oracle
from paper_2502_16982_amd import binding, experts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 20


def args(tokens=4, width=64, inner=32, top=2, n=8, dtype=1, act=0, gate=FAKE, **over):
    m = binding.muon_matrices
    a = binding.muon_layer(m(gate, width * inner, inner), m(FAKE, width * inner, inner), m(FAKE, inner * width, width), tokens, width, inner, top, n,
                           dtype, act, 0)
    for key, value in over.items():
        setattr(a, key, value)
    return a


def test_bytes_refusals():
    L, out = binding.lib(), C.c_size_t(0)
    assert L.muon_expert_layer_bytes(C.byref(args()), C.byref(out)) == 0 and out.value > 0
    assert L.muon_expert_layer_bytes(C.byref(args(tokens=0)), C.byref(out)) == 0 and out.value > 0
    assert L.muon_expert_layer_bytes(None, C.byref(out)) == -1
    assert L.muon_expert_layer_bytes(C.byref(args()), None) == -1
    for bad in (dict(tokens=-1), dict(top=0), dict(top=65), dict(n=0), dict(n=4097), dict(tokens=(1 << 14) // 2 + 1), dict(width=0), dict(inner=0),
                dict(width=(1 << 17) + 1), dict(inner=(1 << 17) + 1), dict(act=2), dict(act=-1), dict(reserved=1)):
        assert L.muon_expert_layer_bytes(C.byref(args(**bad)), C.byref(out)) == -1, bad
    assert L.muon_expert_layer_bytes(C.byref(args(dtype=2)), C.byref(out)) == -2


def test_call_refusals():
    L = binding.lib()
    need = binding.muon_expert_layer_bytes(args())

    def call(a, x=FAKE, stride=64, expert=FAKE, size=8, weights=FAKE, out=FAKE, ws=FAKE, nbytes=need):
        return L.muon_expert_layer(C.byref(a) if a is not None else None, x, stride, expert, size, weights, out, ws, nbytes, None)

    a = args()
    assert call(None) == -1
    assert call(a, x=None) == call(a, expert=None) == call(a, out=None) == call(a, stride=63) == call(a, size=2) == -1
    assert call(a, ws=None) == call(a, nbytes=need - 1) == -4
    assert call(a, x=FAKE + 1) == call(a, expert=FAKE + 4) == call(a, weights=FAKE + 2) == call(a, out=FAKE + 1) == call(a, ws=FAKE + 16) == -7
    m = binding.muon_matrices
    assert call(args(up=m(None, 2048, 32))) == call(args(down=m(None, 2048, 64))) == -1
    assert call(args(up=m(FAKE, 2048, 31))) == call(args(down=m(FAKE, 2048, 63))) == call(args(down=m(FAKE, -1, 64))) == -1
    far = (1 << 24) + 1
    assert call(args(up=m(FAKE, 2048, far))) == call(args(down=m(FAKE, 2048, far))) == -1
    g = args()
    g.gate = m(FAKE, 2048, far)
    assert call(g) == -1
    g.gate = m(FAKE, 2048, 31)
    assert call(g) == -1
    g.gate = m(FAKE + 1, 2048, 32)
    assert call(g) == -7
    assert call(args(up=m(FAKE + 1, 2048, 32))) == call(args(down=m(FAKE + 1, 2048, 64))) == -7
    assert call(args(tokens=0), x=None, expert=None, out=None, ws=None, nbytes=0) == 0       # nothing to do


def test_binding_refuses():
    x, up, down = torch.zeros(3, 16), torch.zeros(4, 16, 8), torch.zeros(4, 8, 16)
    e = torch.zeros(3, 2, dtype=torch.int64)
    for call in (lambda: experts.layer(x, up, down, e),                                        # not on a GPU
                 lambda: experts.layer(x, up, down, e[0]), lambda: experts.layer(x, up, down, e.float()),
                 lambda: experts.layer(x, up, down, e.T)):
        with pytest.raises(binding.MuonError):
            call()
    with pytest.raises(ValueError):
        experts.layer(x, up, down, e, activation="tanh")


def test_plans(tmp_path):
    """Runs cover the summed axis, sections do not overlap, launches stay below 2^32 threads, over the whole range of sizes."""
    exe = str(tmp_path / "layer_plan")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "layer_plan_main.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and "ok" in out.stdout, out.stdout + out.stderr


def test_oracle():
    rng = np.random.default_rng(0)
    x, up, gate, down = (rng.standard_normal(s) for s in ((2, 3), (2, 3, 4), (2, 3, 4), (2, 4, 3)))
    expert, w = np.array([[0, 1], [-1, 2]]), np.array([[0.25, 2.0], [1.0, 1.0]])
    out, bound = layer_oracle.layer(x, up, down, expert, w, gate)
    z = [x[0] @ gate[e] for e in (0, 1)]
    want = sum(c * ((z[e] / (1 + np.exp(-z[e])) * (x[0] @ up[e])) @ down[e]) for e, c in ((0, 0.25), (1, 2.0)))
    assert np.allclose(out[0], want, rtol=1e-14) and (out[1] == 0).all() and (bound >= 0).all()
    t = torch.from_numpy(x[0]) @ torch.from_numpy(gate[0])
    assert np.allclose(layer_oracle.act("silu", t.numpy()), torch.nn.functional.silu(t).numpy(), rtol=1e-14)
    out, _ = layer_oracle.layer(x, up, down, expert, None, None, "relu")
    assert np.allclose(out[0], sum(np.maximum(x[0] @ up[e], 0) @ down[e] for e in (0, 1)), rtol=1e-14)


def test_launches(tmp_path):
    """No axis of a launch holds 2^32 threads, at the largest sizes that are taken either."""
    exe = str(tmp_path / "layer_grid")
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "layer_grid_main.cpp"), "-o", exe], check=True)
    out = subprocess.run([exe], capture_output=True, text=True)
    assert out.returncode == 0 and "ok" in out.stdout, out.stdout + out.stderr
