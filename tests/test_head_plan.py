"""The head's planner on the CPU, built with the address and undefined-behaviour sanitizers: sections, pieces, tiles and splits of many
sizes, and the forms of launch that the GPU tests mean to run."""
import os
import subprocess

import pytest

from tests.head_routes import ROUTES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2502_16982_amd", "csrc")


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("head_plan") / "head_plan")
    proc = subprocess.run(["g++", "-O1", "-g", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-fsanitize=address,undefined",
                           "-fno-sanitize-recover=all", f"-I{CSRC}", os.path.join(ROOT, "tests", "head_plan_main.cpp"),
                           os.path.join(CSRC, "head_plan.cpp"), "-o", out], capture_output=True, text=True)
    assert proc.returncode == 0, proc.stderr[-2000:]
    return out


def test_plans_hold_what_the_launches_rely_on(program):
    proc = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert proc.returncode == 0, (proc.stdout + proc.stderr)[-3000:]


def test_the_gpu_tests_take_every_form_of_launch(program):
    seen = {"logits": set(), "hidden": set(), "weight": set()}
    for tokens, vocab, width in ROUTES:
        for f32 in (0, 1):
            text = subprocess.run([program, str(tokens), str(vocab), str(width), str(f32)], capture_output=True, text=True, check=True).stdout
            for line in text.splitlines():
                name, *fields = line.split()
                f = dict(x.split("=") for x in fields)
                form = f["tile"] + ("a" if f["alone"] == "1" else "") + ("s" if int(f["splits"]) > 1 else "") + ("q" if int(f["quarters"]) else "")
                seen[name].add(form)
    assert {"128", "128a", "256", "256q"} <= seen["logits"], seen
    assert {"128as", "128s", "256", "256s"} <= seen["hidden"], seen
    assert {"128", "128a", "128as", "128s", "256", "256q", "256s"} <= seen["weight"], seen
