"""Values whose squares do not add up within fp32 while the squares of their distances from the mean do."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg

pytestmark = pytest.mark.gpu


# positions and channels of a group, images: a lane holds all of the group's values, or some
@pytest.mark.parametrize("S,D,I", [(16, 8, 1 << 15), (16, 8, 3), (64, 8, 3), (16, 4, 1 << 15), (20000, 8, 1)])
def test_squares_that_overflow(S, D, I):
    C, n = 64, S * D
    gen = np.random.default_rng(3)
    x = torch.randn(1, I, S, C, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    # mean and spread such that sum x^2 = 4.2e38, past the largest fp32 value, of which the distances are 28 %
    size = (4.2e38 / n) ** 0.5
    values = torch.from_numpy(0.85 * size + 0.53 * size * gen.choice([-1.0, 1.0], (S, D))).bfloat16()
    x[0, I // 2, :, D:2 * D] = values.cuda()
    v = values.double().numpy()
    mean, var = v.mean(), v.var()
    assert (v * v).sum() > 3.5e38 and var * n < 3e38
    y, m, r = kavg.kavg_group_norm(x, None, None, C // D, stats=True)
    m, r, got = float(m[0, I // 2, 1]), float(r[0, I // 2, 1]), y[0, I // 2, :, D:2 * D].double().cpu().numpy()
    K = 300 * 2.0 ** -24                                     # (sums as layers_reference.py bounds them)
    assert abs(m - mean) <= K * np.abs(v).max() and abs(r * var ** 0.5 - 1) <= 4 * K
    assert (np.abs(got - (v - mean) / var ** 0.5) <= 2.0 ** -8 * np.abs(got) + 12 * K).all()
