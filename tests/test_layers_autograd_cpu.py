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
