"""What a group gives depends on its own values alone, to the last bit: not on those of the groups, images and learners beside it."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_gpu_group_norm import DTYPES, _inputs

pytestmark = pytest.mark.gpu


# several groups, images and learners in a wavefront; half a pack and two elements of one per group; an image that is read twice
@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(2, 3, 16, 64, 8), (2, 8, 4, 16, 2), (4, 4, 4, 8, 1), (1, 4, 64, 64, 16), (1, 2, 128, 48, 8), (1, 1, 20000, 64, 8), (1, 1, 20000, 40, 10)],
                         ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("beside", [96.0, 3e4])
def test_values_beside_a_group(shape, dtype, beside):
    J, I, S, C, G = shape
    x, dy, w, b = _inputs(shape, dtype, 41, offset=0.1)
    near = torch.zeros(J, I, 1, G, 1, dtype=torch.bool, device="cuda")
    near[0, 0, 0, 0] = True                                  # (the group that stays as it is)
    near[J - 1, I - 1, 0, G // 2] = True
    near = near.expand(J, I, S, G, C // G).reshape(x.shape)
    both = []
    for at in (x, torch.where(near, x, x + beside)):
        y, mean, rstd = kavg.kavg_group_norm(at, w, b, G, activation=kavg.KAVG_ACT_SILU, stats=True)
        dx, _, _ = kavg.kavg_group_norm_backward(dy, at, mean, rstd, w, b, G, activation=kavg.KAVG_ACT_SILU)
        own = near[:, :, 0].view(J, I, G, -1)[..., 0]
        both.append((y[near], mean[own], rstd[own], dx[near]))
    for p, q in zip(*both):
        assert torch.equal(p, q)
