"""layers.mlp and layers.linear without a GPU: the two calls of the library are replaced by plain ones of the same interface and the same demands on strides."""
import pytest
import torch

from paper_2110_00625_amd import kavg, layers

ACT = {kavg.KAVG_ACT_NONE: lambda z: z, kavg.KAVG_ACT_RELU: torch.relu, kavg.KAVG_ACT_SILU: lambda z: z * torch.sigmoid(z)}


def refuse(ok):
    if not ok:
        raise kavg.KavgError(kavg.KAVG_EINVAL, "strides or shapes")


def lies_together(t):
    return t.shape[-1] < 2 or t.stride(-1) == 1


@pytest.fixture
def kept(monkeypatch):
    """Whether each product was asked for its pre-activations."""
    asked = []

    def linear(x, weight, bias=None, activation=kavg.KAVG_ACT_NONE, residual=None, pre=False):
        refuse(x.dim() == weight.dim() and x.dim() in (2, 3) and x.shape[-1] == weight.shape[-1] and x.dtype is weight.dtype)
        refuse(lies_together(x) and (lies_together(weight) or lies_together(weight.mT)))
        refuse(bias is None or lies_together(bias))
        z = x @ weight.mT
        z = z if bias is None else z + bias[..., None, :]
        refuse(residual is None or (residual.shape == z.shape and lies_together(residual)))
        asked.append(pre)
        y = ACT[activation](z)
        y = (y if residual is None else y + residual).contiguous()
        return (y, z) if pre else y

    def backward(dz, x, weight, activation=kavg.KAVG_ACT_NONE, pre=None, out=None, dweight=None, dbias=None):
        refuse(all(lies_together(t) for t in (dz, x)) and (lies_together(weight) or lies_together(weight.mT)))
        dx = dz @ weight
        if activation == kavg.KAVG_ACT_RELU:
            dx = dx * (pre > 0)
        elif activation == kavg.KAVG_ACT_SILU:
            s = torch.sigmoid(pre)
            dx = dx * (s + pre * s * (1 - s))
        return None if out is False else dx, None if dweight is False else dz.mT @ x, None if dbias is False else dz.sum(-2)
    monkeypatch.setattr(kavg, "kavg_linear", linear)
    monkeypatch.setattr(kavg, "kavg_linear_backward", backward)
    return asked


def chain(seed=0, lead=()):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *shape: torch.randn(*lead, *shape, generator=g, dtype=torch.float64).requires_grad_()  # noqa: E731
    return [(normal(6, 4), normal(6)), (normal(5, 6), None), (normal(3, 5), normal(3))]


def test_pre_activations_are_kept_where_a_gradient_can_follow(kept):
    x = torch.ones(2, 4, dtype=torch.float64)
    for activation, keeps in (("silu", [True, True, False]), ("relu", [True, True, False]), (None, [False] * 3)):
        layers.mlp(x, chain(), activation)
        assert kept == keeps
        kept.clear()
    for without in (torch.no_grad(), torch.inference_mode()):
        with without:
            layers.mlp(x, chain(), "silu")
        assert kept == [False] * 3
        kept.clear()
    layers.mlp(x, [(w.detach(), None) for w, _ in chain()], "silu")
    assert kept == [False] * 3
