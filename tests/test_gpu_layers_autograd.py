"""The layers as differentiable functions, and the learners of residual blocks that are made of them.

Gradients of the whole net in fp32 against autograd in 64 bits: each of the dozen operators on the way is off by at most
R.K = 300 * 2^-24 of its terms' magnitudes, and a sum of the norm's backward pass can cancel terms of about four times its size, so
12 * 4 * R.K < 1e-3 of a gradient's length."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg, layers, residual
from tests import layers_reference as R


def test_patches_are_the_neighbours():
    X = torch.arange(2 * 4 * 5 * 3).float().view(2, 4, 5, 3)
    p = residual.patches(X, torch.float32).view(2, 4, 5, 3, 3, 3)
    for i, j, kh, kw in ((0, 0, 0, 0), (3, 4, 2, 2), (1, 2, 1, 1), (2, 0, 0, 2)):
        assert torch.equal(p[:, i, j, kh, kw], X[:, (i + kh - 1) % 4, (j + kw - 1) % 5])


def test_unknown_activation():
    with pytest.raises(kavg.KavgError) as e:
        layers.group_norm(torch.zeros(1, 1, 8), None, None, 2, activation="tanh")
    assert e.value.code == kavg.KAVG_EINVAL


def _normal(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("act,code", [(None, kavg.KAVG_ACT_NONE), ("relu", kavg.KAVG_ACT_RELU), ("silu", kavg.KAVG_ACT_SILU)])
def test_group_norm_gives_the_backward_pass_of_the_library(dtype, act, code):
    x, w, b = _normal(1, 2, 3, 40, 24).to(dtype).requires_grad_(), _normal(2, 2, 24).requires_grad_(), _normal(3, 2, 24).requires_grad_()
    opt = dict(drop=0.2, seed=4, site=5)
    y = layers.group_norm(x, w, b, 4, eps=1e-4, activation=act, **opt)
    want, mean, rstd = kavg.kavg_group_norm(x.detach(), w.detach(), b.detach(), 4, eps=1e-4, activation=code, stats=True, **opt)
    assert torch.equal(y, want)
    # whole, of a sum (strides of zero), and of a transposed use (another order)
    for dy, loss in ((_normal(6, *y.shape).to(dtype), None), (torch.ones_like(y), lambda y: y.sum()),
                     (torch.arange(40, device="cuda").to(dtype)[:, None].expand_as(y).contiguous(),
                      lambda y: (y.transpose(2, 3) * torch.arange(40, device="cuda").to(dtype)).sum())):
        got = torch.autograd.grad(y if loss is None else loss(y), (x, w, b), dy if loss is None else None, retain_graph=True)
        back = kavg.kavg_group_norm_backward(dy, x.detach(), mean, rstd, w.detach(), b.detach(), 4, activation=code, **opt)
        assert all(torch.equal(p, q) for p, q in zip(got, back))
    with torch.no_grad():
        assert torch.equal(layers.group_norm(x, w, b, 4, eps=1e-4, activation=act, **opt), want)
    z = x.detach().requires_grad_()
    assert torch.equal(torch.autograd.grad(layers.group_norm(z, None, None, 4).float().square().sum(), z)[0].isfinite().all(), torch.tensor(True, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_dropout_gives_the_backward_pass_of_the_library(dtype):
    x, r = _normal(1, 2, 30, 24).to(dtype).requires_grad_(), _normal(2, 2, 30, 24).to(dtype).requires_grad_()
    y = layers.dropout(x, 0.3, 7, site=2, residual=r)
    assert torch.equal(y, kavg.kavg_dropout(x.detach(), 0.3, 7, site=2, residual=r.detach()))
    dy = _normal(3, 2, 30, 24).to(dtype)
    dx, dr = torch.autograd.grad(y, (x, r), dy, retain_graph=True)
    assert torch.equal(dr, dy) and torch.equal(dx, kavg.kavg_dropout_backward(dy, 0.3, 7, site=2))
    dx, dr = torch.autograd.grad(y.sum(), (x, r))
    assert torch.equal(dr, torch.ones_like(dr)) and torch.equal(dx, kavg.kavg_dropout_backward(torch.ones_like(x), 0.3, 7, site=2))
    only = layers.dropout(x.detach(), 0.3, 7, residual=r)
    assert torch.equal(torch.autograd.grad(only, r, dy)[0], dy)


def _plain_losses(net, params, x, y):
    """ResidualLearners.losses in 64 bits on the CPU, from the definitions."""
    P, B, S, _ = x.shape

    def norm(h, w, b):
        hg = h.view(P, B, S, net.groups, -1)
        hg = hg - hg.mean((2, 4), keepdim=True)
        z = (hg / (hg.square().mean((2, 4), keepdim=True) + 1e-5).sqrt()).view(h.shape) * w[:, None, None] + b[:, None, None]
        return z * torch.sigmoid(z)

    def product(h, w):
        return torch.matmul(h.reshape(P, B * S, -1), w).view(P, B, S, -1)
    h = product(x, params["w0"])
    for t in range(net.blocks):
        a = product(norm(h, params["gamma%d" % t], params["beta%d" % t]), params["w%d" % (t + 1)])
        h = h + a * torch.from_numpy(R.keep_factors(tuple(a.shape), net.drop, net.seed + net.step, t))
    logits = torch.matmul(norm(h, params["gamma"], params["beta"]).mean(2), params["head"]) + params["b"][:, None]
    return -torch.log_softmax(logits, 2).gather(2, y[:, :, None].long()).mean((1, 2))


@pytest.mark.gpu
@pytest.mark.parametrize("side,channels,groups", [(6, 32, 4), (5, 21, 7), (9, 40, 5)])
def test_gradients_of_the_residual_learners(side, channels, groups):
    P, B, classes = 3, 4, 5
    net = residual.ResidualLearners(P, 27, channels, 2, groups, classes, 0.1, 0.5, drop=0.2, seed=9, dtype=torch.float32)
    net.replicas += 0.1 * _normal(1, *net.replicas.shape)                      # (the learners differ)
    x = residual.patches(_normal(2, P * B, side, side, 3), torch.float32).view(P, B, side * side, 27)
    y = torch.arange(P * B, device="cuda").view(P, B) % classes
    losses, grads = net.gradients(x, y)
    leaves = {k: p.detach().cpu().double().requires_grad_() for k, p in net.params.items()}
    want = _plain_losses(net, leaves, x.cpu().double(), y.cpu())
    assert np.allclose(losses.cpu(), want.detach(), rtol=1e-3, atol=0)
    for got, (name, leaf) in zip(grads, leaves.items()):
        g = torch.autograd.grad(want.sum(), leaf, retain_graph=True)[0]
        assert got.shape == g.shape and float((got.cpu().double() - g).norm()) <= 1e-3 * float(g.norm()), name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_residual_learners_learn(dtype):
    curve = residual.train(P=4, K=2, B=16, side=8, channels=32, blocks=2, groups=4, rounds=12, N=512, dtype=dtype)
    assert np.isfinite(curve).all() and np.mean(curve[-3:]) < np.mean(curve[:3])
