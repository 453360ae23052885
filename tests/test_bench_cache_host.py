"""The benchmark's tuning cache is for the pointwise kernels: it holds as long as their sources do, whatever else is in the library."""
import os
import shutil
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def bench(tmp_path, monkeypatch):
    monkeypatch.syspath_prepend(ROOT)
    sys.modules.pop("bench", None)
    import bench as b
    assert os.path.abspath(b.__file__) == os.path.join(ROOT, "bench.py")
    shutil.copytree(os.path.join(ROOT, "paper_2109_00170_b200", "csrc"), tmp_path / "paper_2109_00170_b200" / "csrc")
    monkeypatch.setattr(b, "ROOT", str(tmp_path))
    yield b
    sys.modules.pop("bench", None)


@pytest.mark.parametrize("name,same", [("alcs_norm.cu", True), ("alcs_mx4.cu", True), ("alcs_mx4_product.cu", True), ("alcs_dense.h", True), ("alcs_call.c", True),
                                       ("alcs_conv2d.cu", True), ("alcs_tc.cu", False), ("alcs_tc.cuh", False), ("alcs_gather.cu", False), ("alcs_device.cu", False),
                                       ("alcs_kernels.cuh", False)])
def test_which_sources_the_cache_depends_on(bench, tmp_path, name, same):
    before = bench.kernel_source_hash()
    with open(tmp_path / "paper_2109_00170_b200" / "csrc" / name, "a") as f:
        f.write("// changed\n")
    assert (bench.kernel_source_hash() == before) == same
