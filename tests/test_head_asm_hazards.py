"""The head's products read LDS fragments from inline assembly with hand-placed waits: the generated gfx950 assembly is checked for any
instruction that touches the destination of an LDS read which no wait has retired (no GPU needed)."""
import os
import subprocess

import pytest

from paper_2502_16982_amd import build
from tests import asm_lds_hazards as hz


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "head.s"
    cmd = [build.hipcc_path(), *build.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, "kernels_head.hip"), "-o", str(out)]
    proc = subprocess.run(cmd, capture_output=True, text=True, cwd=str(out.parent))
    assert proc.returncode == 0, proc.stderr[-2000:]
    return hz.split_kernels(out.read_text())


def test_products_wait_for_every_lds_read_they_use(kernels):
    logits = {k: v for k, v in kernels.items() if "head_logits" in k}
    products = {k: v for k, v in kernels.items() if "head_product" in k}
    assert len(logits) == 9 and len(products) == 12          # {256, 128, 128 alone} x {none, f16, fp32}; x {plain, K-major} x {whole, parts}
    for name, lines in {**logits, **products}.items():
        assert any("ds_read_b128" in t or "ds_read_b64_tr_b16" in t for _, t in lines)
        assert hz.check_kernel(lines) == [], name
    for name, lines in products.items():
        assert sum("ds_read_b64_tr_b16" in t for _, t in lines) >= 16, name
        assert not any("scratch_" in t for _, t in lines), name          # no spills


def test_no_packed_fp32(kernels):
    for name, lines in kernels.items():
        assert not any(t.startswith(("v_pk_add_f32", "v_pk_mul_f32", "v_pk_fma_f32")) for _, t in lines), name


def test_a_loosened_wait_is_caught(kernels):
    """Sensitivity: the first wait after a transposing read, loosened to one that lets fifteen reads be outstanding."""
    name, lines = next((k, v) for k, v in kernels.items() if "head_productILi128" in k or "head_product_kernelILi128" in k)
    first = next(i for i, (_, t) in enumerate(lines) if "ds_read_b64_tr_b16" in t)
    at = next(i for i in range(first, len(lines)) if lines[i][1] == "s_waitcnt lgkmcnt(0)")
    loose = [*lines[:at], (lines[at][0], "s_waitcnt lgkmcnt(15)"), *lines[at + 1:]]
    assert hz.check_kernel(loose) != [], name
