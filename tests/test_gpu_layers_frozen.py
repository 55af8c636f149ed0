"""Group norm whose parameters, or some of them, want no gradient."""
import pytest
import torch

from paper_2110_00625_amd import kavg, layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(2, 3, 40, 24, 4), (1, 2, 5000, 64, 8), (1, 2, 40, 1031, 1)], ids=str)
def test_gradients_that_nobody_asks_for(shape, dtype):
    J, I, S, C, G = shape
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(J, I, S, C, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w, b = (torch.randn(J, C, generator=gen, device="cuda") for _ in range(2))
    opt = dict(activation=kavg.KAVG_ACT_SILU, drop=0.1, seed=3)
    _, mean, rstd = kavg.kavg_group_norm(x, w, b, G, stats=True, **opt)
    whole = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G, **opt)
    for kw in (dict(dweight=False), dict(dbias=False), dict(dweight=False, dbias=False)):
        got = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G, **opt, **kw)
        assert torch.equal(got[0], whole[0])
        for k, name in ((1, "dweight"), (2, "dbias")):
            assert got[k] is None if name in kw else torch.equal(got[k], whole[k])
    x.requires_grad_()
    opt["activation"] = "silu"
    layers.group_norm(x, w, b, G, **opt).backward(dy)
    assert torch.equal(x.grad, whole[0])
    b.requires_grad_()
    layers.group_norm(x.detach(), w, b, G, **opt).backward(dy)
    assert torch.equal(b.grad, whole[2]) and w.grad is None
