"""bench.py quotes a stored traffic figure while the sources of the kernels that it was measured on are unchanged: files that the
layer is not built from do not take the figure away, and every file that it is built from does."""
import os
import shutil

import pytest

import bench

CSRC = os.path.join("paper_2501_10375_amd", "csrc")


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A copy of the kernel sources and the profiles that the benchmark looks at instead of the repository's."""
    shutil.copytree(os.path.join(bench.ROOT, CSRC), tmp_path / CSRC)
    shutil.copytree(os.path.join(bench.ROOT, "profiles"), tmp_path / "profiles")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    return tmp_path / CSRC


def append(path):
    with open(path, "a") as f:
        f.write("// another line\n")


@pytest.mark.parametrize("name", ["another_operator.hip", "another_operator.h", "products_api.hip", "products_tiles.h", "quantize_fp8.hip"])
def test_sources_beside_the_layer_leave_its_figure(tree, name):
    before = bench.kernel_source_digest()
    append(tree / name)
    assert bench.kernel_source_digest() == before


@pytest.mark.parametrize("name", ["ffn_bf16.hip", "ffn_bf16_decode.hip", "ffn_f32.hip", "route.hip", "permute.hip", "moe_api.hip",
                                  "grouped_gemm_bf16.h", "hand_out.h", "bf16_utils.h", "route_device.h", "moe_internal.h"])
def test_sources_of_the_layer_count(tree, name):
    before = bench.kernel_source_digest()
    append(tree / name)
    assert bench.kernel_source_digest() != before
    assert bench.read_traffic("mixtral_prefill_T4096_gemm1")[0] is None


def test_the_stored_figures_are_those_of_the_sources(tree):
    """The layer's kernels have not changed since the counters were read (where they do, the counters have to be read again)."""
    figure, source = bench.read_traffic("mixtral_prefill_T4096_gemm1")
    assert figure is not None, source
