"""Group norm and dropout as differentiable torch functions: kavg_group_norm and kavg_dropout of the library with their backward
passes.  What autograd keeps of a group norm is its input and two statistics per group, of a dropout nothing: the mask is drawn
again from (drop, seed, site), where seed is not the index_seed of a context (its minibatch indices come from the same generator).
A program that writes its own backward pass calls `kavg` instead, which can also write into given tensors (a learner's gradient
vector, x itself)."""
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
