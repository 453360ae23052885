"""Group norm at the edges of its ranges: clusters with blocks that have no pixels."""
import pytest

import test_gpu_norm as norm

pytestmark = pytest.mark.gpu


# 49 and 25 pixels in clusters of 8 blocks of 7 and 4: the last block has none (all but the fp32 one of one group of 1024 channels, which takes two passes)
@pytest.mark.parametrize("dtype,act", [("f32", "none"), ("f32", "silu"), ("f16", "relu"), ("bf16", "silu")])
@pytest.mark.parametrize("shape", [(1, 7, 7, 512, 1), (2, 7, 7, 1024, 1), (1, 7, 7, 1024, 4), (3, 7, 7, 2048, 8), (1, 5, 5, 2048, 2), (5, 5, 5, 512, 1)],
                         ids=lambda s: "x".join(map(str, s)))
def test_blocks_without_pixels(alcs, shape, dtype, act):
    norm.test_forward_and_backward(alcs, shape, dtype, act)
