"""The workspace of the head's losses on the CPU: one for a call serves every smaller call, and a limit never makes it larger."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_16982_amd", "csrc")


def test_a_workspace_serves_smaller_calls_and_limits_hold(tmp_path):
    out = str(tmp_path / "head_workspace")
    proc = subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", f"-I{CSRC}", os.path.join(ROOT, "tests", "head_workspace_main.cpp"),
                           os.path.join(CSRC, "head_plan.cpp"), "-o", out], capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr[-2000:]
    proc = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, (proc.stdout + proc.stderr)[-3000:]


@pytest.mark.parametrize("tokens,vocab,width,dtype", [(300, 131072, 4096, 1), (4096, 131072, 4096, 1), (512, 100003, 2048, 0)])
def test_a_limit_never_makes_the_answer_larger(tokens, vocab, width, dtype):
    from paper_2502_16982_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2502_16982_amd import build
        build.build_library()
    h = binding.muon_head(None, None, width, width, tokens, vocab, width, dtype, 0)
    whole = binding.muon_head_workspace_bytes(h, 1, 3)
    for limit in (1, whole // 2, whole - 256, whole):
        assert binding.muon_head_workspace_bytes(h, 1, 3, limit) <= whole
    smaller = binding.muon_head(None, None, width, width, tokens * 3 // 4, vocab, width, dtype, 0)
    assert binding.muon_head_workspace_bytes(smaller, 1, 3) <= whole
