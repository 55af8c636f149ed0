"""What the differentiable layers hand back to autograd, with the library's calls replaced by plain torch on the CPU."""
import pytest
import torch

from paper_2110_00625_amd import kavg, layers


@pytest.fixture
def plain_dropout(monkeypatch):
    """Twice every second element."""
    def dropped(x, drop, seed, site=0, residual=None):
        y = torch.where(torch.arange(x.numel()).view(x.shape) % 2 == 0, 2 * x, torch.zeros(()))
        return y if residual is None else y + residual
    monkeypatch.setattr(kavg, "kavg_dropout", dropped)
    monkeypatch.setattr(kavg, "kavg_dropout_backward", dropped)


def test_dropout_without_a_residual(plain_dropout):
    x = torch.ones(3, 4, requires_grad=True)
    layers.dropout(x, 0.5, 1).sum().backward()
    assert torch.equal(x.grad, torch.tensor([2.0, 0.0]).repeat(3, 2))


def test_dropout_of_what_needs_no_gradient(plain_dropout):
    x, residual = torch.ones(3, 4), torch.ones(3, 4, requires_grad=True)
    layers.dropout(x, 0.5, 1, residual=residual).sum().backward()
    assert x.grad is None and torch.equal(residual.grad, torch.ones(3, 4))
    x.requires_grad_()
    layers.dropout(x, 0.5, 1, residual=torch.ones(3, 4)).sum().backward()
    assert torch.equal(x.grad, torch.tensor([2.0, 0.0]).repeat(3, 2))


@pytest.mark.parametrize("wanted", [(True, True, True), (True, False, False), (True, True, False), (True, False, True), (False, True, True), (False, False, True)], ids=str)
def test_group_norm_asks_for_the_gradients_that_are_wanted(monkeypatch, wanted):
    asked = []

    def forward(x, weight, bias, groups, stats=False, **options):
        return (x.clone(), torch.zeros(2, groups), torch.ones(2, groups)) if stats else x.clone()

    def backward(dy, x, mean, rstd, weight, bias, groups, dweight=None, dbias=None, **options):
        asked.append((dweight is not False, dbias is not False))
        return dy, None if dweight is False else torch.ones_like(weight), None if dbias is False else torch.ones_like(bias)
    monkeypatch.setattr(kavg, "kavg_group_norm", forward)
    monkeypatch.setattr(kavg, "kavg_group_norm_backward", backward)
    x, w, b = torch.ones(2, 3, 8), torch.ones(8), torch.zeros(8)
    for t, want in zip((x, w, b), wanted):
        t.requires_grad_(want)
    layers.group_norm(x, w, b, 2).sum().backward()
    assert asked == [wanted[1:]]
    for t, want in zip((x, w, b), wanted):
        assert (t.grad is not None) == want
