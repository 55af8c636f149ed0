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


def plain(x, parts, activation, residual):
    h = x
    for i, (w, b) in enumerate(parts):
        h = h @ w.mT if w.dim() == 2 else (h.reshape(h.shape[0], -1, h.shape[-1]) @ w.mT).view(*h.shape[:-1], -1)
        if b is not None:
            h = h + (b if w.dim() == 2 else b.view(b.shape[0], *[1] * (h.dim() - 2), -1))
        h = ACT[layers.ACTIVATIONS[activation]](h) if i + 1 < len(parts) else h
    return h if residual is None else h + residual


def apart(t):
    """The values of t in a tensor of no stride of 1."""
    return torch.stack((t, torch.full_like(t, float("nan"))), -1).detach()[..., 0]


@pytest.mark.parametrize("sets,dims", [(None, ()), (None, (7,)), (None, (2, 7)), (3, ()), (3, (7,)), (3, (2, 7))], ids=str)
def test_x_of_any_dimensions_and_any_strides(kept, sets, dims):
    """A single sample without rows, too; operands and residuals in any order, weights and biases in every second place of a tensor."""
    lead = () if sets is None else (sets,)
    g = torch.Generator().manual_seed(5)
    x, r, dy = (torch.randn(*lead, *dims, n, generator=g, dtype=torch.float64) for n in (4, 3, 3))
    turn = lambda t: t.transpose(-1, 0).contiguous().transpose(-1, 0)  # noqa: E731
    parts = [tuple(None if p is None else p.detach() for p in layer) for layer in chain(1, lead)]
    want_leaves = [t.clone().requires_grad_() for t in [x, r] + [p for layer in parts for p in layer if p is not None]]
    it = iter(want_leaves[2:])
    want = plain(want_leaves[0], [tuple(None if p is None else next(it) for p in layer) for layer in parts], "silu", want_leaves[1])
    want_grads = torch.autograd.grad(want, want_leaves, dy)
    for move in (torch.clone, turn, apart):
        leaves = [move(t).requires_grad_() for t in [x, r] + [p for layer in parts for p in layer if p is not None]]
        it = iter(leaves[2:])
        got = layers.mlp(leaves[0], [tuple(None if p is None else next(it) for p in layer) for layer in parts], "silu", residual=leaves[1])
        assert got.shape == want.shape and torch.allclose(got, want)
        for a, b in zip(torch.autograd.grad(got, leaves, dy), want_grads):
            assert a.shape == b.shape and torch.allclose(a, b)
    assert layers.linear(x, parts[0][0]).shape == (*lead, *dims, 6)


def test_what_does_not_fit_is_refused(kept):
    w, b = torch.ones(6, 4), torch.ones(6)
    for call in (lambda: layers.linear(torch.ones(()), w), lambda: layers.linear(torch.ones(3), w), lambda: layers.linear(torch.ones(2, 4), w[None]), lambda: layers.linear(torch.ones(4), w[None]),
                 lambda: layers.linear(torch.ones(2, 4), w[0]), lambda: layers.linear(torch.ones(2, 4), w[None, None]), lambda: layers.mlp(torch.ones(2, 4), [(None, b)]),
                 lambda: layers.linear(torch.ones(2, 4), w, 1.0), lambda: layers.linear(torch.ones(2, 4), w, torch.ones(())),
                 lambda: layers.mlp(torch.ones(2, 4), [(w, b), (b, b)]), lambda: layers.mlp(torch.ones(2, 4), [(w, b), (w[None, :, :].expand(2, 6, 4), b)]),
                 lambda: layers.linear(torch.ones(4), w, residual=torch.ones(1, 6))):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == kavg.KAVG_EINVAL
