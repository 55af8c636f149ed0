"""Group norm of many vectors and many images of a few positions, whose lanes fill the device several times over, against the 64-bit
forms of layers_reference.py."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_gpu_group_norm import DTYPES, _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 1024, 1, 1024, 16), (4, 1025, 1, 512, 8), (1, 2048, 2, 256, 8), (2, 1100, 9, 96, 8), (1, 9000, 1, 91, 7), (1, 3000, 6, 33, 3)],
                         ids=lambda s: "-".join(map(str, s)))
def test_many_small_images(shape, dtype):
    for act, drop in ((kavg.KAVG_ACT_SILU, 0.1), (kavg.KAVG_ACT_RELU, 0.0)):
        x, dy, w, b = _inputs(shape, dtype, shape[1])
        _check(x, dy, w, b, shape[4], act, drop)
