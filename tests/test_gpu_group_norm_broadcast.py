"""Group norm of inputs whose images share memory (strides of 0, overlapping images), with channels that fill no pack, against the
64-bit forms of layers_reference.py."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_gpu_group_norm import DTYPES, _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 9, 1, 1, 1), (1, 64, 1, 5, 1), (1, 3, 1, 3, 1), (2, 5, 1, 7, 7), (2, 9, 7, 1, 1), (3, 2, 2, 3, 3), (1, 5, 40, 9, 3),
                                   (1, 2, 20000, 3, 1)], ids=lambda s: "-".join(map(str, s)))
def test_images_that_are_one(shape, dtype):
    """x and dy are one image of a learner, or one of all learners."""
    x, dy, w, b = _inputs(shape, dtype, 21)
    for act, drop in ((kavg.KAVG_ACT_SILU, 0.2), (kavg.KAVG_ACT_NONE, 0.0)):
        for sets in (slice(None), slice(0, 1)):
            one, grad = (t[sets, :1].expand_as(t) for t in (x, dy))
            _check(one.contiguous(), grad.contiguous(), w, b, shape[4], act, drop, make=lambda t: t[sets, :1].clone().expand_as(t))


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 4, 1, 3, 1), (2, 3, 1, 7, 7), (1, 9, 2, 1, 1), (2, 5, 33, 5, 1)], ids=lambda s: "-".join(map(str, s)))
def test_images_that_overlap(shape, dtype):
    """Image i + 1 begins an element behind image i, as windows of one line of values do."""
    J, I, S, C, G = shape
    _, _, w, b = _inputs(shape, dtype, 22)
    views = {}
    for k in range(2):
        line = torch.randn(J + I + S * C - 2, generator=torch.Generator(device="cuda").manual_seed(k), device="cuda").to(dtype)
        view = line.as_strided((J, I, S, C), (1, 1, C, 1))
        dense = view.contiguous()
        views[dense.data_ptr()] = dense, view
    (x, _), (dy, _) = views.values()
    _check(x, dy, w, b, G, kavg.KAVG_ACT_SILU, 0.2, make=lambda t: views[t.data_ptr()][1])
