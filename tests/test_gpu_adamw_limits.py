"""AdamW steps at the limits of their numbers: denominators that are subnormal in fp32, or whose reciprocal is."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_gpu_adamw import OPTIONS, check_step, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("eps", (1e-37, 1e-38, 2e-39, 1e-45, 1e-60, 1e-300, 8e37, 1e38, 1e60))
def test_any_eps(eps, bits, dtype):
    """Of gradients of 0 the moments are 0, the denominator is eps and the change 0; where a gradient's square is 0 in fp32 the denominator is eps and the change is
    not; others do not see a small eps, and a large one lets through what large moments leave."""
    p, g = normal(1, 2000), normal(2, 2000, scale=1e-2)
    p[::2] = 0
    g[300:600] = 0
    if eps > 1e-70:
        g[600:900] *= 1e-28
    g[1024:] *= 1e18
    plan = kavg.AdamW([p], bits=bits)
    before = p.clone()
    for step in (1, 2):
        check_step(plan, [g.to(dtype)], step, options=dict(OPTIONS, eps=eps))
        if step == 1:
            decay = 1 - OPTIONS["lr"] * OPTIONS["weight_decay"]
            assert (plan.params[0][300:600].double() - before[300:600].double() * decay).abs().max() <= 2.0 ** -23 * before.abs().max()


def test_an_eps_of_zero_is_the_formula_s():
    """0 / 0 where nothing has moved yet, the gradient's sign elsewhere."""
    p, g = torch.zeros(600, device="cuda"), normal(2, 600)
    g[100:200] = 0
    kavg.AdamW([p]).step([g], 1, lr=0.5, eps=0.0, weight_decay=0.0)
    assert torch.isnan(p[100:200]).all()
    # (the moments' and the rates' roundings, some ten of 2^-24)
    moved = torch.cat((p[:100], p[200:])) + 0.5 * torch.sign(torch.cat((g[:100], g[200:])))
    assert moved.abs().max() <= 0.5 * 20 * 2.0 ** -24
