"""Products as differentiable functions on the device, of operands whose last dimension does not lie together and of samples without rows: the bits of the same
calls with whole tensors."""
import pytest
import torch

from paper_2110_00625_amd import layers
from tests.test_gpu_learner_layers import normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("lead,dims", [((), ()), ((), (9,)), ((3,), ()), ((3,), (2, 5))], ids=str)
def test_any_strides(lead, dims, dtype):
    def every_second(t):
        return torch.stack((t, torch.full_like(t, float("nan"))), -1)[..., 0]
    x, r, dy = normal(1, *lead, *dims, 24, dtype=dtype), normal(2, *lead, *dims, 16, dtype=dtype), normal(3, *lead, *dims, 16, dtype=dtype)
    parts = [normal(4, *lead, 40, 24, scale=0.2), normal(5, *lead, 40), normal(6, *lead, 16, 40, scale=0.2)]
    results = []
    for move in (torch.clone, every_second):
        leaves = [move(t).requires_grad_() for t in (x, r, *parts)]
        a, b, w, u, v = leaves
        y = layers.mlp(a, [(w, u), (v, None)], "silu", residual=b)
        assert y.shape == r.shape
        results.append([y, *torch.autograd.grad(y, leaves, dy)])
        with torch.no_grad():
            assert torch.equal(layers.mlp(a, [(w, u), (v, None)], "silu", residual=b), y)
    assert all(torch.equal(p, q) for p, q in zip(*results))
