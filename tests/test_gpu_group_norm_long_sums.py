"""Sums of many terms: statistics of long images, gradients of the parameters of many images and of images that one lane goes through for
long.  The gradient's terms are of one sign and size, so that a running fp32 sum loses the same way at every step: the error of n
additions one after the other is up to n 2^-25 of the sum, against K of layers_reference.py, which allows for 256 of them."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import layers_reference as R

pytestmark = pytest.mark.gpu


def _check(x, groups, value):
    """dbias and dweight of a constant gradient without an activation: value * count, value * sum of xh; x [1][I][S][C] may be broadcast."""
    _, I, S, C = x.shape
    w, b = torch.ones(1, C, device="cuda"), torch.zeros(1, C, device="cuda")
    _, mean, rstd = kavg.kavg_group_norm(x, w, b, groups, stats=True)
    dy = torch.full((C,), value, dtype=x.dtype, device="cuda").expand(x.shape)
    g = float(dy[0, 0, 0, 0])
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, groups)
    del dx
    each = x.stride(1) == 0                                  # (one image, many times)
    xh = torch.zeros(C, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(xh)
    for i in range(0, 1 if each else I, 4096):
        k = min(4096, I - i) if not each else 1
        v = x[0, i:i + k].double().view(k, S, groups, -1)
        var, m = torch.var_mean(v, (1, 3), correction=0)
        assert ((mean[0, i:i + k].double() - m).abs() <= R.K * v.abs().amax((1, 3))).all()
        assert ((rstd[0, i:i + k].double() * (var + 1e-5).sqrt() - 1).abs() <= R.K).all()
        v = v - mean[0, i:i + k].double()[:, None, :, None]
        v = (v * rstd[0, i:i + k].double()[:, None, :, None]).view(-1, C)
        xh += v.sum(0)
        size += v.abs().sum(0)
    times = I if each else 1
    assert (db[0].double() / (g * I * S) - 1).abs().max() <= R.K
    assert ((dw[0].double() - g * times * xh).abs() <= R.K * g * times * size).all()


def _x(shape, dtype):
    x = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    x[..., 0] = x[..., 0].abs() + 1                          # (a channel whose xh is of one sign)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 200000, 1, 64, 8), (1, 300000, 2, 24, 3), (1, 100000, 1, 65, 5), (1, 30000, 5, 513, 1)], ids=lambda s: "-".join(map(str, s)))
def test_many_images(shape, dtype):
    _check(_x(shape[:4], dtype), shape[4], 0.1)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("images,positions", [(342, 4096), (350, 10007)])
def test_long_images_of_groups_that_no_tile_takes(images, positions, dtype):
    _check(_x((1, 1, positions, 513), dtype).expand(1, images, positions, 513), 1, 0.1)


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("images,positions,channels,groups", [(512, 65536, 64, 8), (1100, 40000, 33, 3)])
def test_long_images_on_tiles(images, positions, channels, groups, dtype):
    _check(_x((1, 1, positions, channels), dtype).expand(1, images, positions, channels), groups, 0.12850189)
