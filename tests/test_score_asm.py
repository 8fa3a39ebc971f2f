"""The generated gfx950 assembly of the scores', the clipping's and the few tokens' layer's kernels: LDS reads that are waited for, no packed fp32,
registers that stay registers (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2502_16982_amd import build
from tests import asm_lds_hazards as hz


@pytest.fixture(scope="module", params=["kernels_score.hip", "kernels_clip.hip", "kernels_layer.hip"])
def assembly(request, tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "kernels.s"
    cmd = [build.hipcc_path(), *build.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, request.param), "-o", str(out)]
    proc = subprocess.run(cmd, capture_output=True, text=True, cwd=str(out.parent))
    assert proc.returncode == 0, proc.stderr[-2000:]
    return request.param, out.read_text()


def test_products_wait_for_every_lds_read_they_use(assembly):
    """The tiles' reads of LDS are written in assembly and waited for by hand."""
    name, text = assembly
    if name != "kernels_score.hip":
        pytest.skip("no LDS reads of its own")
    kernels = {k: v for k, v in hz.split_kernels(text).items() if "score_logits" in k or "score_grad" in k}
    assert len(kernels) == 18
    for k, lines in kernels.items():
        assert sum("v_mfma" in line for _, line in lines) > 0
        assert hz.check_kernel(lines) == [], k


def test_no_packed_fp32(assembly):
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", assembly[1])


def test_spills(assembly):
    """None, but for a few registers around the epilogues of the 256-wide tiles."""
    found = dict(re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", assembly[1], re.S))
    assert found
    for name, size in found.items():
        wide = "score_logits_kernelILi256E" in name or "score_grad_kernelILi256E" in name
        assert int(size) <= (16 if wide else 0), (name, size)
