"""The workspace of the head's losses on the CPU: one for a call serves every smaller call, and a limit never makes it larger."""
import os
import subprocess

import pytest

from tests.head_pieces import PIECES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_16982_amd", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("head_workspace") / "head_workspace")
    proc = subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", f"-I{CSRC}", os.path.join(ROOT, "tests", "head_workspace_main.cpp"),
                           os.path.join(CSRC, "head_plan.cpp"), "-o", out], capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr[-2000:]
    return out


def test_a_workspace_serves_smaller_calls_and_limits_hold(program):
    proc = subprocess.run([program], capture_output=True, text=True, timeout=300)
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


def test_the_gpu_tests_take_every_form_of_pieces(program):
    """Pieces' gradients of W that are added to and kept: in runs of K, in 256-wide tiles, with the last round in quarters."""
    for name, (tokens, vocab, width, f32, limit) in PIECES.items():
        text = subprocess.run([program, *map(str, (tokens, vocab, width, int(f32), limit))], capture_output=True, text=True, check=True).stdout
        first, whole, _ = text.splitlines()
        assert int(first.split()[1]) >= 3, text
        f = whole.split()
        tile, splits, quarters = int(f[1]), int(f[3]), int(f[5])
        assert (splits > 1) == ("runs of K" in name) and (tile == 256) == ("256" in name) and (quarters > 0) == ("quarters" in name), (name, text)


@pytest.mark.parametrize("call,pieces,of", [((20000, 32768, 1024, 0, 300_000_000), 16, 1280), ((20000, 32768, 1024, 0, 0), 3, 6912),
                                            ((1_000_000, 50257, 768, 0, 400_000_000), 652, 1536)])
def test_pieces_are_as_large_as_their_splits_allow(program, call, pieces, of):
    """Room is made for the sums of the runs of K that a plan has, a few megabytes of what any plan might have."""
    text = subprocess.run([program, *map(str, call)], capture_output=True, text=True, check=True).stdout
    assert text.splitlines()[0] == f"pieces {pieces} of {of}", text
