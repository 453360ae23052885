"""Sources of the dense operators' kernels.  They start while the kernel before them still writes (programmatic dependent launch): none of their loads may go
through the read-only path, which is for memory that nobody writes as long as the kernel runs.  And lanes have to be together where an instruction is .aligned."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2109_00170_b200", "csrc")


@pytest.mark.parametrize("name", ["alcs_norm.cu", "alcs_mx4.cu", "alcs_mx4_product.cu", "alcs_dense.h"])
def test_no_load_through_the_read_only_path(name):
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    assert "wait_for_previous" in code
    assert not re.findall(r"__ldg\s*\(|\.nc\b|__restrict__", code)


@pytest.mark.parametrize("name", ["alcs_norm.cu", "alcs_mx4_product.cu", "alcs_dense.h"])
def test_lanes_meet_before_a_barrier_of_the_cluster(name):
    """barrier.cluster.*.aligned: all lanes of a warp together, and nothing but a __syncwarp directly before it says so (barriers of the block and full-mask
    exchanges are followed by branches)."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//[^\n]*", "", f.read())
    barriers = re.findall(r"([^;{}]*[;{}])\s*asm volatile\(\"barrier\.cluster[^;]*\.aligned", code)
    assert all(b.strip() == "__syncwarp();" for b in barriers) and len(barriers) == code.count("barrier.cluster")
    assert len(barriers) == (2 if name == "alcs_dense.h" else 0)
