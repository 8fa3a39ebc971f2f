"""Registers of the head's kernels that go to memory, from the generated gfx950 assembly (no GPU needed)."""
import os
import re
import subprocess

from paper_2502_16982_amd import build


def test_no_kernel_of_the_head_spills_more_than_three_registers(tmp_path):
    """None does but the 256-wide logits with fp32 logits kept, which spills 12 bytes per lane around its epilogue."""
    out = tmp_path / "head.s"
    cmd = [build.hipcc_path(), *build.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, "kernels_head.hip"), "-o", str(out)]
    proc = subprocess.run(cmd, capture_output=True, text=True, cwd=str(tmp_path))
    assert proc.returncode == 0, proc.stderr[-2000:]
    found = dict(re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_private_segment_fixed_size (\d+)", out.read_text(), re.S))
    assert sum("head_logits" in k for k in found) == 9 and sum("head_product" in k for k in found) == 12
    for name, size in found.items():
        assert int(size) <= (12 if "head_logits_kernelILi256ELi2ELb1ELb1E" in name else 0), (name, size)
