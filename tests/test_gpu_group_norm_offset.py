"""Gradients of groups that lie far from zero against their spread, with the statistics given.  The formula takes x and the mean by their
difference alone, which fp32 has within 2^-24 of itself; so the bounds of layers_reference.py hold with x - mean in the place of x."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import layers_reference as R
from tests.test_gpu_group_norm import _inputs, _np, _within

pytestmark = pytest.mark.gpu


# held by a workgroup, read twice, channels that fill no pack (both), groups that no tile takes
@pytest.mark.parametrize("shape", [(2, 3, 64, 64, 8), (1, 2, 5000, 64, 8), (1, 1, 16383, 320, 32), (1, 3, 30, 7, 1), (1, 1, 20000, 33, 3), (1, 2, 40, 1031, 1)],
                         ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("act,drop", [(kavg.KAVG_ACT_NONE, 0.0), (kavg.KAVG_ACT_SILU, 0.1)])
@pytest.mark.parametrize("offset", [100.0, 10000.0])
def test_gradient_far_from_zero(shape, act, drop, offset):
    J, I, S, C, G = shape
    x, dy, w, b = _inputs(shape, torch.float32, 31, offset=0.0)
    x = x + offset
    xg = _np(x).reshape(J, I, S, G, C // G)
    mean = xg.mean(axis=(2, 4))
    rstd = 1 / np.sqrt(((xg - mean[:, :, None, :, None]) ** 2).mean(axis=(2, 4)) + 1e-5)
    mean, rstd = (torch.from_numpy(t).float().cuda() for t in (mean, rstd))
    m = np.broadcast_to(_np(mean)[:, :, None, :, None], xg.shape).reshape(x.shape)
    dy = dy + torch.from_numpy(_np(x) - m).float().cuda()                # (a gradient that goes with x)
    f = R.keep_factors(tuple(x.shape), drop, 7, 1)
    got = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G, activation=act, drop=drop, seed=7, site=1)
    wants, bounds = R.group_norm_backward(_np(dy), _np(x) - m, 0 * _np(mean), _np(rstd), _np(w), _np(b), G, act, f)
    for g, want, bound in zip(got, wants, bounds):
        _within(g, want, bound)
