"""Group norm, dropout and products as differentiable torch functions: kavg_group_norm, kavg_dropout and kavg_linear of the library with
their backward passes.  What autograd keeps of a group norm is its input and two statistics per group, of a dropout nothing: the mask is drawn
again from (drop, seed, site), where seed is not the index_seed of a context (its minibatch indices come from the same generator); of
products their inputs, their weights and, where an activation follows, what it was given.
A program that writes its own backward pass calls `kavg` instead, which can also write into given tensors (a learner's gradient
vector, x itself)."""
import math

import torch
from torch.autograd.function import once_differentiable

from . import kavg

ACTIVATIONS = {None: kavg.KAVG_ACT_NONE, "relu": kavg.KAVG_ACT_RELU, "silu": kavg.KAVG_ACT_SILU}


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, groups, eps, options):
        if not any(ctx.needs_input_grad):
            return kavg.kavg_group_norm(x, weight, bias, groups, eps=eps, **options)
        y, mean, rstd = kavg.kavg_group_norm(x, weight, bias, groups, eps=eps, stats=True, **options)
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        ctx.groups, ctx.options = groups, options
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        # (a gradient can have any strides, that of a sum for example zeros)
        wanted = ctx.needs_input_grad
        dx, dweight, dbias = kavg.kavg_group_norm_backward(dy.contiguous(), *ctx.saved_tensors, ctx.groups, dweight=None if wanted[1] else False,
                                                           dbias=None if wanted[2] else False, **ctx.options)
        return dx if wanted[0] else None, dweight, dbias, None, None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, options):
        ctx.options = options
        return kavg.kavg_dropout(x, residual=residual, **options)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dx = kavg.kavg_dropout_backward(dy.contiguous(), **ctx.options) if ctx.needs_input_grad[0] else None
        return dx, dy if ctx.needs_input_grad[1] else None, None


def group_norm(x, weight, bias, groups, eps=1e-5, activation=None, drop=0.0, seed=0, site=0):
    """Group norm of x [sets, images, positions, channels] with weight, bias [sets, channels] (x of three dimensions: one set),
    then the activation (None, "relu", "silu"), then dropout where drop > 0; as in kavg.kavg_group_norm."""
    if activation not in ACTIVATIONS:
        raise kavg.KavgError(kavg.KAVG_EINVAL, "activation %r is none of %s" % (activation, list(ACTIVATIONS)))
    return _GroupNorm.apply(x, weight, bias, groups, eps, {"activation": ACTIVATIONS[activation], "drop": drop, "seed": seed, "site": site})


def dropout(x, drop, seed, site=0, residual=None):
    """residual + dropout(x), as in kavg.kavg_dropout."""
    return _Dropout.apply(x, residual, {"drop": drop, "seed": seed, "site": site})


def _shape(x, weight):
    """x [sets, .., inputs] or [.., inputs] as [sets, rows, inputs] or [rows, inputs]."""
    if x.dim() < weight.dim() - 1 or (weight.dim() == 3 and x.shape[0] != weight.shape[0]):
        raise kavg.KavgError(kavg.KAVG_EINVAL, "x of %s and weights of %s" % (tuple(x.shape), tuple(weight.shape)))
    rows = math.prod(x.shape[weight.dim() - 2:-1])
    return x.reshape(x.shape[0], rows, x.shape[-1]) if weight.dim() == 3 else x.reshape(rows, x.shape[-1])


def _together(t, either=False):
    """t, or a copy of it where its last dimension (either: one of its last two) does not lie together."""
    if t is None or t.shape[-1] < 2 or t.stride(-1) == 1 or (either and (t.shape[-2] < 2 or t.stride(-2) == 1)):
        return t
    return t.contiguous()


class _Products(torch.autograd.Function):
    """residual + (.. act(act(x W_1^T + b_1) W_2^T + b_2) ..) W_n^T + b_n.  parameters: W_1, b_1, .., W_n, b_n."""

    @staticmethod
    def forward(ctx, x, residual, activation, recorded, *parameters):
        weights, biases = parameters[::2], parameters[1::2]
        # (recorded: whether gradients are recorded around the call; in here they never are)
        last, wanted, kept, inputs, used = len(weights) - 1, recorded and any(ctx.needs_input_grad), [], [], []
        h = x
        for i, (w, b) in enumerate(zip(weights, biases)):
            w = w.to(x.dtype)                                        # (float32 weights of bfloat16 activations)
            inputs.append(h)
            used.append(w)
            if i == last:
                h = kavg.kavg_linear(h, w, b, residual=residual)
            elif wanted and activation != kavg.KAVG_ACT_NONE:
                h, pre = kavg.kavg_linear(h, w, b, activation=activation, pre=True)
                kept.append(pre)
            else:
                h = kavg.kavg_linear(h, w, b, activation=activation)
        if wanted:
            ctx.save_for_backward(*inputs, *used, *kept)
            ctx.activation, ctx.n, ctx.types = activation, len(weights), [w.dtype for w in weights]
        return h

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        n, saved, wanted = ctx.n, ctx.saved_tensors, ctx.needs_input_grad
        inputs, weights, kept = saved[:n], saved[n:2 * n], saved[2 * n:]
        dz, grads = dy.contiguous(), [None] * (2 * n)
        lowest = min([i for i in range(n) if wanted[4 + 2 * i] or wanted[5 + 2 * i]] + [0 if wanted[0] else n])
        for i in range(n - 1, lowest - 1, -1):
            inner = wanted[0] if i == 0 else i > lowest
            dx, dw, db = kavg.kavg_linear_backward(
                dz, inputs[i], weights[i], activation=ctx.activation if i else kavg.KAVG_ACT_NONE, pre=kept[i - 1] if i and kept else None, out=None if inner else False,
                dweight=None if wanted[4 + 2 * i] else False, dbias=None if wanted[5 + 2 * i] else False)
            grads[2 * i], grads[2 * i + 1] = None if dw is None else dw.to(ctx.types[i]), db
            dz = dx
        return dz if wanted[0] else None, dy if wanted[1] else None, None, None, *grads


def mlp(x, layers, activation="silu", residual=None):
    """residual + the last of n products, with the activation ("relu", "silu" or None) between them: x [sets, .., inputs] with layers
    [(weight, bias), ..], weight [sets, outputs, inputs], bias [sets, outputs] (float32) or None; or all of them without sets.  Any strides will do (what
    lies in no order that kavg.kavg_linear takes is copied).  Weights are of x's type, or float32 with bfloat16 activations (rounded in the call).  The activations' derivatives are taken in the epilogues of the
    products of the backward pass; gradients of float32 weights are float32."""
    if activation not in ACTIVATIONS:
        raise kavg.KavgError(kavg.KAVG_EINVAL, "activation %r is none of %s" % (activation, list(ACTIVATIONS)))
    layers = [tuple(layer) for layer in layers]
    if not layers or not all(len(layer) == 2 and isinstance(layer[0], torch.Tensor) and layer[0].dim() in (2, 3) and
                             (layer[1] is None or (isinstance(layer[1], torch.Tensor) and layer[1].dim())) for layer in layers):
        raise kavg.KavgError(kavg.KAVG_EINVAL, "%d layers of a weight (of two or three dimensions) and a bias" % len(layers))
    layers = [(_together(weight, either=True), _together(bias)) for weight, bias in layers]
    flat = _together(_shape(x, layers[0][0]))
    outputs = layers[-1][0].shape[-2]
    shape = (*x.shape[:-1], outputs)
    if residual is not None:
        if residual.shape != shape:
            raise kavg.KavgError(kavg.KAVG_EINVAL, "a residual of %s for %s" % (tuple(residual.shape), shape))
        residual = _together(residual.reshape(*flat.shape[:-1], outputs))
    return _Products.apply(flat, residual, ACTIVATIONS[activation], torch.is_grad_enabled(), *[p for layer in layers for p in layer]).view(shape)


def linear(x, weight, bias=None, residual=None):
    """residual + x W^T + bias, as in mlp (and in kavg.kavg_linear, which a program without gradients calls for an activation behind it)."""
    return mlp(x, [(weight, bias)], None, residual)
