"""Products as differentiable functions, and learners that train with them and with AdamW.

Gradients of a chain in fp32 against autograd in 64 bits: a product of K terms is off by at most 2 (K + 1) 2^-24 of its terms' magnitudes, here
K <= 100, and an activation by less; a gradient passes three products and two activations, so that 5 * 2 * 101 * 2^-24 < 1e-4 of the magnitudes, which
are less than ten times a gradient's length: 1e-3 of that.  In bf16 each of the chain's roundings is half a step, 2^-8 of its value: six of them on
the way, of magnitudes that are less than ten times a gradient's length in the worst case, and each rounding's sign is as good as random: 6 * 2^-8 * 2 = 0.05."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg, layers, residual
from tests import layers_reference as R

pytestmark = pytest.mark.gpu


def normal(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def plain_mlp(x, chain, activation, add):
    h = x
    for i, (w, b) in enumerate(chain):
        h = h @ w.transpose(-1, -2)
        if b is not None:
            h = h + (b if w.dim() == 2 else b.reshape(b.shape[0], *([1] * (h.dim() - 2)), -1))
        if i + 1 < len(chain):
            h = torch.relu(h) if activation == "relu" else torch.nn.functional.silu(h) if activation == "silu" else h
    return h if add is None else h + add


@pytest.mark.parametrize("dtype,near", ((torch.float32, 1e-3), (torch.bfloat16, 0.05)), ids=("f32", "bf16"))
@pytest.mark.parametrize("activation", (None, "relu", "silu"))
@pytest.mark.parametrize("sets,widths", [(None, (40, 24)), (3, (40, 24)), (2, (33, 100, 7)), (None, (16, 64, 48, 16)), (2, (24, 96, 24))], ids=str)
def test_chains(sets, widths, activation, dtype, near):
    lead = () if sets is None else (sets,)
    x = normal(1, *lead, 5, 6, widths[0], dtype=dtype).requires_grad_()
    chain = [(normal(10 + i, *lead, b, a, scale=a ** -0.5).requires_grad_(), None if i == 1 else normal(20 + i, *lead, b, scale=0.3).requires_grad_())
             for i, (a, b) in enumerate(zip(widths, widths[1:]))]
    add = normal(2, *lead, 5, 6, widths[-1], dtype=dtype).requires_grad_()
    y = layers.mlp(x, chain, activation, residual=add)
    leaves = [x, add] + [p for layer in chain for p in layer if p is not None]
    double = [t.detach().double().requires_grad_() for t in leaves]
    it = iter(double[2:])
    plain_chain = []
    for w, b in chain:
        plain_chain.append((next(it), next(it) if b is not None else None))
    wide = [(w if sets is None else w[:, None], b) for w, b in plain_chain]
    want = plain_mlp(double[0], wide, activation, double[1])
    assert y.shape == want.shape and float((y.double() - want).detach().norm()) <= near * float(want.detach().norm())
    dy = normal(3, *y.shape, dtype=dtype)
    got = torch.autograd.grad(y, leaves, dy)
    for g, e, leaf in zip(got, torch.autograd.grad(want, double, dy.double()), leaves):
        assert g.dtype is leaf.dtype and g.shape == leaf.shape and float((g.double() - e).norm()) <= near * float(e.norm())
    with torch.no_grad():
        assert torch.equal(layers.mlp(x, chain, activation, residual=add), y)


def test_a_gradient_of_a_sum_and_of_frozen_parts():
    """Gradients with strides of zero, and only those that are asked for, of whatever layer."""
    x, w1, w2, b1 = normal(1, 30, 16), normal(2, 24, 16), normal(3, 8, 24), normal(4, 24)
    every = [x, w1, b1, w2]
    whole = [t.clone().requires_grad_() for t in every]
    full = torch.autograd.grad(layers.mlp(whole[0], [(whole[1], whole[2]), (whole[3], None)]).sum(), whole)
    for k in range(4):
        part = [t.clone().requires_grad_(i == k) for i, t in enumerate(every)]
        got = torch.autograd.grad(layers.mlp(part[0], [(part[1], part[2]), (part[3], None)]).sum(), part[k])[0]
        assert torch.equal(got, full[k]) or k == 2
        assert float((got - full[k]).abs().max()) <= 1e-5 * float(full[k].abs().max())
    none = layers.mlp(torch.empty(2, 0, 3, 16, device="cuda"), [(normal(6, 2, 24, 16), normal(7, 2, 24)), (normal(8, 2, 8, 24), None)])
    assert none.shape == (2, 0, 3, 8)
    r = normal(5, 30, 8).requires_grad_()
    assert torch.equal(torch.autograd.grad(layers.linear(x, normal(6, 8, 16), residual=r).sum(), r)[0], torch.ones_like(r))


def test_weights_in_the_replicas_and_turned():
    rows = normal(1, 3, 24 * 16 + 24 + 3, scale=0.2)
    for w in (rows[:, :384].view(3, 24, 16), rows[:, :384].view(3, 16, 24).transpose(1, 2)):
        leaf, b = w.detach().requires_grad_(), rows[:, 384:408].detach().requires_grad_()
        x = normal(2, 3, 4, 5, 16, dtype=torch.bfloat16).requires_grad_()
        y = layers.linear(x, leaf, b)
        dx, dw, db = torch.autograd.grad(y, (x, leaf, b), torch.ones_like(y))
        want = kavg.kavg_linear_backward(torch.ones(3, 20, 24, dtype=torch.bfloat16, device="cuda"), x.detach().view(3, 20, 16), w.bfloat16())
        assert torch.equal(dx.view(3, 20, 16), want[0]) and torch.equal(dw, want[1]) and torch.equal(db, want[2]) and dw.dtype is torch.float32


def test_refusals():
    x, w, b = normal(1, 5, 8), normal(2, 6, 8), normal(3, 6)
    for call in (lambda: layers.mlp(x, [], "silu"), lambda: layers.mlp(x, [(w, b, b)]), lambda: layers.mlp(x, [(w, b)], "tanh"), lambda: layers.linear(x, w, residual=x),
                 lambda: layers.linear(x, w[None].expand(2, 6, 8)), lambda: layers.linear(x[:, :7], w), lambda: layers.mlp(x, [(w, b), (w, b)])):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == kavg.KAVG_EINVAL


def test_a_backward_pass_in_a_graph_beside_an_eager_one():
    """Leaves whose eager graph is still alive are trained by a captured backward pass of their detached twins; replays follow the inputs."""
    x, w, b = normal(1, 40, 16), normal(2, 24, 16).requires_grad_(), normal(3, 24).requires_grad_()
    alive = layers.linear(x.clone(), w, b)                                    # (its graph is kept)

    def gradients(x, w, b):
        w, b = w.detach().requires_grad_(), b.detach().requires_grad_()
        return torch.autograd.grad(layers.mlp(x, [(w, b)]).square().sum(), (w, b))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        gradients(x, w, b)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gradients(x, w, b)
    for k in range(4):
        x.copy_(normal(10 + k, 40, 16))
        graph.replay()
        torch.cuda.synchronize()
        for g, e in zip(out, gradients(x, w, b)):
            assert torch.equal(g, e)
    assert torch.isfinite(torch.autograd.grad(alive.sum(), b)[0]).all()


def _plain_losses(net, params, x, y):
    """ResidualLearners.losses with hidden layers in 64 bits on the CPU, from the definitions."""
    P, B, S, _ = x.shape

    def norm(h, w, b):
        hg = h.reshape(P, B, S, net.groups, -1)
        hg = hg - hg.mean((2, 4), keepdim=True)
        z = (hg / (hg.square().mean((2, 4), keepdim=True) + 1e-5).sqrt()).view(h.shape) * w[:, None, None] + b[:, None, None]
        return z * torch.sigmoid(z)

    def product(h, w):
        return torch.matmul(h.reshape(P, B * S, -1), w).view(P, B, S, -1)
    h = product(x, params["w0"])
    for t in range(net.blocks):
        a = product(norm(h, params["gamma%d" % t], params["beta%d" % t]), params["w%d" % (t + 1)])
        h = h + a * torch.from_numpy(R.keep_factors(tuple(a.shape), net.drop, net.seed + net.step, t))
        z = product(h, params["U%d" % t].transpose(1, 2)) + params["u%d" % t][:, None, None]
        h = h + product(z * torch.sigmoid(z), params["V%d" % t].transpose(1, 2)) + params["v%d" % t][:, None, None]
    logits = torch.matmul(norm(h, params["gamma"], params["beta"]).mean(2), params["head"]) + params["b"][:, None]
    return -torch.log_softmax(logits, 2).gather(2, y[:, :, None].long()).mean((1, 2))


@pytest.mark.parametrize("side,channels,groups,hidden", [(6, 32, 4, 64), (5, 21, 7, 30)])
def test_gradients_of_learners_with_hidden_layers(side, channels, groups, hidden):
    """As the learners without them; two products and an activation more a block, so that twenty operators at the same bound stay below 2e-3."""
    P, B, classes = 3, 4, 5
    net = residual.ResidualLearners(P, 27, channels, 2, groups, classes, 0.1, 0.5, drop=0.2, seed=9, dtype=torch.float32, hidden=hidden)
    net.replicas += 0.1 * normal(1, *net.replicas.shape)
    x = residual.patches(normal(2, P * B, side, side, 3), torch.float32).view(P, B, side * side, 27)
    y = torch.arange(P * B, device="cuda").view(P, B) % classes
    losses, grads = net.gradients(x, y)
    leaves = {k: p.detach().cpu().double().requires_grad_() for k, p in net.params.items()}
    want = _plain_losses(net, leaves, x.cpu().double(), y.cpu())
    assert np.allclose(losses.cpu(), want.detach(), rtol=2e-3, atol=0)
    for got, (name, leaf) in zip(grads, leaves.items()):
        g = torch.autograd.grad(want.sum(), leaf, retain_graph=True)[0]
        assert got.shape == g.shape and float((got.cpu().double() - g).norm()) <= 2e-3 * float(g.norm()), name


@pytest.mark.parametrize("bits", (8, 32))
@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
def test_learners_run_with_adamw(dtype, bits):
    """Rounds of products, norms, dropout, AdamW steps and meta steps together: they run, every learner's parameters move and are averaged."""
    curve = residual.train(P=4, K=2, B=16, side=8, channels=32, blocks=2, groups=4, rounds=6, N=512, dtype=dtype, hidden=48, adamw=bits, lr=0.003)
    assert len(curve) == 6 and np.isfinite(curve).all()


def test_a_local_step_is_the_step_of_its_gradients():
    net = residual.ResidualLearners(2, 27, 32, 1, 4, 5, 0.01, 0.5, drop=0.0, seed=3, dtype=torch.float32, hidden=40, adamw=32)
    x = residual.patches(normal(2, 8, 6, 6, 3), torch.float32).view(2, 4, 36, 27)
    y = torch.arange(8, device="cuda").view(2, 4) % 5
    before = {k: p.clone() for k, p in net.params.items()}
    _, grads = net.gradients(x, y)
    net.local_step(x, y)
    for (name, p), g, decay in zip(net.params.items(), grads, net.decay):
        # the first step: m / (1 - beta1) = g, sqrt(v / (1 - beta2)) = |g|, but for roundings of the moments and of 1 - beta (some 2^-20 of the change)
        want = before[name].double() * (1 - 0.01 * decay) - 0.01 * g.double() / (g.double().abs() + 1e-8)
        # (gradients in the size of eps apart, whose squares lose places)
        off = (p.double() - want).abs()
        assert bool((off <= 1e-5 * 0.01 + 2.0 ** -22 * want.abs()).logical_or(g.abs() < 1e-12).all()), name
