"""The kernels of the grouped products issue MFMAs from inline asm like those of the expert GEMMs; the same reading of the built
code holds for them (see test_isa_hazards)."""
import os
import shutil
import subprocess

import pytest

from paper_2501_10375_amd import moe
from test_isa_hazards import OBJDUMP, hazards, parse


def test_built_product_kernels_have_no_mfma_hazard(tmp_path):
    if not os.path.exists(OBJDUMP) or not os.path.exists(moe.LIB_PATH):
        pytest.skip("needs llvm-objdump and the built library")
    shutil.copy(moe.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, stdout=subprocess.DEVNULL)
    kernels = {}
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" in name:
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp_path, check=True, text=True,
                                  stdout=subprocess.PIPE).stdout
            kernels.update(parse(text, "product_gemm_kernel"))
    assert len(kernels) >= 4
    for name, code in kernels.items():
        assert sum(c.mfma for c in code) > 500, name
        assert hazards(code) == [], name
