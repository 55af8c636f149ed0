"""Outputs whose learners, images and positions lie in another order than that of their dimensions, and do not overlap."""
import itertools

import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import AT, lib, norm  # noqa: F401  (lib: the loaded library)

SIZES = {"sets": 2, "images": 3, "positions": 4}


def _strides(order, first=8):
    """(sets, images, positions) for dimensions named from the outermost."""
    at, run = {}, first
    for name in reversed(order):
        at[name] = run
        run *= SIZES[name]
    return tuple(at[k] for k in SIZES)


def _codes(lib, strides):  # noqa: F811
    n, dense, out = norm(**SIZES, channels=8, groups=2), kavg._IMAGES.pack(AT, 96, 32, 8), kavg._IMAGES.pack(AT, *strides)
    return (lib.kavg_group_norm_backward(n, dense, dense, AT, AT, AT, 8, AT, 8, out, AT, 8, AT, 8, None, 0, None))


@pytest.mark.parametrize("order", list(itertools.permutations(SIZES)), ids="-".join)
def test_no_order_is_refused(lib, order):  # noqa: F811
    """(The call ends at its workspace, which is not there.)"""
    strides = _strides(order)
    assert _codes(lib, strides) == kavg.KAVG_ENOMEM
    for k in range(3):                                       # one stride an element too small: something overlaps
        assert _codes(lib, tuple(s - (i == k) for i, s in enumerate(strides))) == kavg.KAVG_EINVAL
    assert _codes(lib, (0, 0, 0)) == kavg.KAVG_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(2, 3, 40, 24, 3), (2, 2, 5000, 64, 8), (3, 2, 33, 21, 7), (2, 3, 20, 1031, 1), (4, 30, 4, 16, 2)], ids=str)
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))), ids=str)
def test_results_in_any_order(shape, dtype, order):
    J, I, S, C, G = shape
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(J, I, S, C, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w, b = (torch.randn(J, C, generator=gen, device="cuda") for _ in range(2))
    sizes, back = [(J, I, S)[k] for k in order], [order.index(k) for k in range(3)] + [3]
    opt = dict(activation=kavg.KAVG_ACT_SILU, drop=0.1, seed=9)

    def place():
        return torch.empty(*sizes, C, dtype=dtype, device="cuda").permute(back)
    y, mean, rstd = kavg.kavg_group_norm(x, w, b, G, stats=True, out=place(), **opt)
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G, out=place(), **opt)
    # (another layout of the work where positions do not lie end to end and channels fill no pack: the same to a few roundings)
    exact = C % 8 == 0 or order.index(2) == 2
    for got, want in zip((y, dx), (kavg.kavg_group_norm(x, w, b, G, **opt), kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G, **opt)[0])):
        if exact:
            assert torch.equal(got, want)
        else:
            assert ((got.double() - want.double()).abs() <= 2.0 ** (-7 if dtype is torch.bfloat16 else -14) * (want.double().abs() + 1)).all()
