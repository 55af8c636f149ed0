"""Plain 64-bit forms of the products of learners' layers and of the AdamW step, and the bounds the kernels are held to.  Shares nothing
with the library.

Products.  A sum of n products in fp32, in whatever order, is off by at most n 2^-24 of the sum of the terms' magnitudes and a product by
2^-24 of itself; twice that allows for additions inside a matrix instruction that cut instead of rounding.  The activation multiplies an error
of z by its slope, 1.1 at most, and adds its own: exp2 and 1/x of the hardware are good for a few 2^-24, and |z| 2^-24 more for the product in front of
the exponential.  A result is rounded once: half a step, finfo.eps / 2 of its value.
"""
import math

import numpy as np
import torch

from tests import layers_reference as R

U = 2.0 ** -24
ACTS = ("none", "relu", "silu")


def rounding(dtype):
    return torch.finfo(dtype).eps / 2


def act(z, kind):
    return torch.relu(z) if kind == "relu" else z * torch.sigmoid(z) if kind == "silu" else z


def slope(z, kind):
    if kind == "relu":
        return (z > 0).double()
    s = torch.sigmoid(z)
    return s + z * s * torch.sigmoid(-z) if kind == "silu" else torch.ones_like(z)


def product(a, b):
    """a [.., M, K] times b [.., N, K] turned, in 64 bits, and the bound on a kernel's fp32 sums."""
    a, b = a.double(), b.double()
    k = a.shape[-1]
    return a @ b.transpose(-1, -2), 2 * (k + 1) * U * (a.abs() @ b.abs().transpose(-1, -2)) + 1e-37


def linear(x, weight, bias, kind, residual, dtype):
    """((y, its bound), (z, its bound))"""
    z, e = product(x, weight)
    if bias is not None:
        z = z + bias.double()[..., None, :]
        e = e + U * z.abs() + U * bias.double().abs()[..., None, :]
    y = act(z, kind)
    e_y = 1.1 * e + (z.abs() * (8 + 2 * z.abs()) * U if kind == "silu" else 0)
    if residual is not None:
        y = y + residual.double()
        e_y = e_y + U * y.abs()
    r = rounding(dtype)
    return (y, e_y * (1 + r) + r * y.abs()), (z, e * (1 + r) + r * z.abs())


def linear_backward(dz, x, weight, kind, pre, dtype):
    """(dx, bound), (dweight, bound), (dbias, bound)"""
    dx, e = product(dz, weight.transpose(-1, -2))
    if kind != "none":
        p = pre.double()
        s = slope(p, kind)
        # (the slope: a few roundings, and the exponential's argument)
        e = e * s.abs() + (dx.abs() * (12 + 2 * p.abs()) * U * (1 + p.abs()) if kind == "silu" else 0) + U * (dx * s).abs()
        dx = dx * s
    r = rounding(dtype)
    dw, e_w = product(dz.transpose(-1, -2), x.transpose(-1, -2))
    db = dz.double().sum(-2)
    e_b = 2 * (dz.shape[-2] + 1) * U * dz.double().abs().sum(-2) + 1e-37
    return (dx, e * (1 + r) + r * dx.abs()), (dw, e_w + U * dw.abs()), (db, e_b)


def close(got, want_and_bound):
    want, bound = want_and_bound
    assert got.shape == want.shape
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), "off by %.3g of the bound" % float((off / bound).max())


# ---- AdamW ----------------------------------------------------------------------------------------------------------

BLOCK, BORDER = 256, 0x3FDDB3D7


def e4m3_values():
    """The values of codes 0 .. 0x7E."""
    return np.array([2.0 ** -9 * c if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(0x7F)])


def scale_of(block):
    """The scale of a block from its definition; block in fp32."""
    block = block[np.isfinite(block)]
    most = np.float64(np.abs(block).max()) if block.size else 0.0
    c = np.float64(np.array([BORDER], dtype=np.uint32).view(np.float32)[0])
    if most == 0:
        return 2.0 ** -126
    k = math.floor(math.log2(most / c)) + 1
    for k in (k - 1, k, k + 1):
        if 2.0 ** (k - 1) * c <= most < 2.0 ** k * c:
            return max(2.0 ** (k - 8), 2.0 ** -126)
    raise AssertionError


def draws(n, seed, site):
    e = np.arange(n, dtype=np.uint64)
    with np.errstate(over="ignore"):
        number = np.uint64(1) + np.uint64(site) * np.uint64(1 << 40) + e // np.uint64(4)
        z = R.mix(np.uint64(seed) + number * np.uint64(0x9E3779B97F4A7C15))
    field = (z >> (np.uint64(16) * (e % np.uint64(4)))) & np.uint64(0xFFFF)
    return (field.astype(np.float64) + 0.5) / 65536


def coded(values, rows, drawn=None):
    """(codes, scales) of fp32 `values` [rows * cols], from the definition: to nearest, or down or up by the draws."""
    table = e4m3_values()
    values = values.reshape(rows, -1)
    cols = values.shape[1]
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // BLOCK)), np.float32)
    for r in range(rows):
        for b in range(scales.shape[1]):
            part = values[r, b * BLOCK:(b + 1) * BLOCK]
            scale = scales[r, b] = scale_of(part)
            q = part.astype(np.float64) / scale
            fine = np.isfinite(q)
            a = np.where(fine, np.abs(q), 0.0)
            low = np.searchsorted(table, a, side="right") - 1
            up = np.minimum(low + 1, 0x7E)
            gap = np.where(up > low, table[up] - table[low], 1.0)
            rest = (a - table[low]) / gap
            if drawn is None:
                code = np.where((rest > 0.5) | ((rest == 0.5) & (low % 2 == 1)), up, low)
            else:
                d = drawn[r * cols + b * BLOCK:r * cols + b * BLOCK + part.size]
                code = np.where(rest.astype(np.float32) + d.astype(np.float32) >= 1, up, low)       # (the sum of two exact numbers, in fp32)
                code = np.where((a > 0) & (code == 0), 1, code)
            codes[r, b * BLOCK:b * BLOCK + part.size] = np.where(fine, code | (0x80 * np.signbit(part)), 0x7F)
    return codes, scales


def adamw(p, g, m, v, step, lr, beta1, beta2, eps, weight_decay, grad_scale=1.0):
    """(p, its bound), and the fp32 moments operation by operation; numpy, p, g, m, v fp32."""
    f = np.float32
    with np.errstate(all="ignore"):
        gs = g * f(grad_scale)
        m32 = m * f(beta1) + gs * f(1 - beta1)
        v32 = v * f(beta2) + (gs * gs) * f(1 - beta2)
        m64, v64 = m32.astype(np.float64), v32.astype(np.float64)
        change = lr / (1 - beta1 ** step) * m64 / (np.sqrt(v64 / (1 - beta2 ** step)) + eps)
        want = p.astype(np.float64) * (1 - lr * weight_decay) - change
    # the decay factor, the rate and the root's factor come rounded, five operations more on the change, three on the parameter
    return (want, 10 * U * np.abs(change) + 4 * U * np.abs(p.astype(np.float64)) + 1e-44), m32, v32
