"""The wait states around the matrix instructions that Muon's products write as assembly (the GEMMs' loop on fp16 operands): as those of the GEMM file."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2512_20953_amd import build
from tests.test_matrix_waits_compile import _check


@pytest.mark.skipif(not shutil.which("hipcc"), reason="no compiler")
def test_wait_states_around_matrix_instructions(tmp_path):
    asm = tmp_path / "muon.s"
    subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "muon.hip"), "-o", str(asm)], check=True, capture_output=True)
    text = asm.read_text()
    kernels = re.findall(r"^(\S*14product_kernel\S+):[^\n]*\n(.*?)\.Lfunc_end", text, re.S | re.M)
    backs = [_check(*k) for k in kernels]
    assert len(backs) == 18 and all(n for n in backs)             # six products in tiles of 256, and of 128 with two ring depths
    assert "v_mfma_f32_16x16x32_f16" in text and "_bf16 a[" not in text
