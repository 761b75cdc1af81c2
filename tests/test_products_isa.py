"""The kernels of the grouped products issue MFMAs from inline asm like those of the expert GEMMs; the same reading of the built
code holds for them (see test_isa_hazards).  In the 8-bit kernel results are vector registers that additions read a few
MFMAs later: 12 wait states behind the eight passes of its only MFMA, which the compiler puts there too when it knows of one."""
import os
import re
import shutil
import subprocess

import pytest

import test_isa_hazards
from paper_2501_10375_amd import moe
from test_isa_hazards import OBJDUMP, hazards, parse


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not os.path.exists(OBJDUMP) or not os.path.exists(moe.LIB_PATH):
        pytest.skip("needs llvm-objdump and the built library")
    tmp = tmp_path_factory.mktemp("isa")
    shutil.copy(moe.LIB_PATH, tmp / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp, check=True, stdout=subprocess.DEVNULL)
    return [subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp, check=True, text=True, stdout=subprocess.PIPE).stdout
            for name in sorted(os.listdir(tmp)) if "gfx950" in name]


def kernels_named(listings, name):
    return {k: code for text in listings for k, code in parse(text, name).items()}


def test_built_bf16_product_kernels_have_no_mfma_hazard(listings):
    kernels = kernels_named(listings, "product_gemm_kernel")
    assert len(kernels) >= 4
    for name, code in kernels.items():
        assert sum(c.mfma for c in code) > 300, name
        assert hazards(code) == [], name


def test_built_fp8_product_kernel_has_no_mfma_hazard(listings, monkeypatch):
    monkeypatch.setattr(test_isa_hazards, "RESULT_WAIT", 12)
    kernels = kernels_named(listings, "product_fp8_kernel")
    assert len(kernels) == 1
    for name, code in kernels.items():
        mfmas = [c for c in code if c.mfma]
        assert len(mfmas) > 100 and {c.op for c in mfmas} == {"v_mfma_f32_16x16x128_f8f6f4"}, name
        assert hazards(code) == [], name


def test_loads_to_lds_do_not_follow_vector_writes_of_their_descriptors(listings):
    """A memory instruction reads a scalar register that a vector instruction wrote five wait states later at the earliest; the
    loads are asm statements, so the compiler does not see to it."""
    loads = 0
    for name in ("product_gemm_kernel", "product_fp8_kernel", "product_small_kernel", "product_small_fp8_kernel"):
        for kernel, code in kernels_named(listings, name).items():
            for n, c in enumerate(code):
                if not (c.op.startswith("buffer_load") and c.text.endswith("lds")):
                    continue
                loads += 1
                lo, hi = map(int, re.search(r"s\[(\d+):(\d+)\]", c.text).groups())
                waited = 0
                for before in reversed(code[max(0, n - 5):n]):
                    if waited >= 5:
                        break
                    m = re.match(r"v_read(?:first)?lane_b32(?:_e64)? s(\d+),", before.text)
                    assert m is None or not lo <= int(m.group(1)) <= hi, (kernel, before.text, c.text)
                    waited += before.wait
    assert loads > 100
