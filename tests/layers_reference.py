"""Plain 64-bit forms of the layers (group norm with activation and dropout, dropout) and of their gradients, in numpy, and the
bounds the kernels are held to.  Shares nothing with the library.

Bounds.  A kernel's fp32 sum of n terms adds at most `CHAIN` of them one after the other in a thread and joins the threads in a
tree: its error is below (CHAIN + 20) 2^-24 times the sum of the terms' magnitudes.  exp and 1/x of the hardware are good for a few
2^-24, with |z| 2^-24 more for the product in front of the exponential.  K below is the sum of these, for sizes where CHAIN <= 256.
An output in bf16 is rounded once more, to nearest: 2^-9 of its value (2^-8 to be clear of a tie that falls the other way).
"""
import numpy as np

ACT_NONE, ACT_RELU, ACT_SILU = 0, 1, 2
K = 300 * 2.0 ** -24


def mix(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    return z ^ (z >> np.uint64(31))


def keep_factors(shape, drop, seed, site):
    """0 where an element is dropped, 1 / (1 - p) elsewhere, from the definition: element by element."""
    e = np.arange(int(np.prod(shape)), dtype=np.uint64)
    with np.errstate(over="ignore"):
        number = np.uint64(1) + np.uint64(site) * np.uint64(1 << 40) + e // np.uint64(4)
        z = mix(np.uint64(seed) + number * np.uint64(0x9E3779B97F4A7C15))
    field = (z >> (np.uint64(16) * (e % np.uint64(4)))) & np.uint64(0xFFFF)
    t = int(np.floor(65536 * drop + 0.5))
    return np.where(field >= t, 65536.0 / (65536 - t) if t < 65536 else 0.0, 0.0).reshape(shape)


def sigmoid(z):
    return 0.5 * (1 + np.tanh(0.5 * z))


def act(z, kind):
    return np.maximum(z, 0) if kind == ACT_RELU else z * sigmoid(z) if kind == ACT_SILU else z


def slope(z, kind):
    if kind == ACT_RELU:
        return (z > 0).astype(np.float64)
    if kind == ACT_SILU:
        return sigmoid(z) * (1 + z * sigmoid(-z))
    return np.ones_like(z)


def grouped(x, groups):
    return x.reshape(x.shape[:-1] + (groups, x.shape[-1] // groups))


def group_norm(x, weight, bias, groups, eps, kind, factors=1.0):
    """x [J][I][S][C] in float64: y, mean, rstd, and the bound on y's error."""
    xg = grouped(x, groups)
    mean = xg.mean(axis=(2, 4), keepdims=True)
    rstd = 1 / np.sqrt(((xg - mean) ** 2).mean(axis=(2, 4), keepdims=True) + eps)
    xh = ((xg - mean) * rstd).reshape(x.shape)
    w, b = weight[:, None, None, :], bias[:, None, None, :]
    z = xh * w + b
    # the mean is off by up to K mean|x|, the variance by up to K of itself and the square of that
    off_mean = (np.abs(xg).mean(axis=(2, 4), keepdims=True) * rstd + 0 * xg).reshape(x.shape)
    bound = K * (np.abs(w) * (np.abs(xh) * (1 + off_mean ** 2 * K) + off_mean) + np.abs(b) + np.abs(z)) * 1.1 * np.abs(factors) + 1e-37
    return act(z, kind) * factors, mean[:, :, 0, :, 0], rstd[:, :, 0, :, 0], bound


def group_norm_backward(dy, x, mean, rstd, weight, bias, groups, kind, factors=1.0):
    """dx, dweight, dbias and their bounds."""
    J, I, S, C = x.shape
    D = C // groups
    r = np.broadcast_to(rstd[:, :, None, :, None], (J, I, S, groups, D)).reshape(x.shape)
    m = np.broadcast_to(mean[:, :, None, :, None], (J, I, S, groups, D)).reshape(x.shape)
    xh = (x - m) * r
    w, b = weight[:, None, None, :], bias[:, None, None, :]
    z = xh * w + b
    da = dy * factors
    dz = da * slope(z, kind)
    h = dz * w

    def over_group(v):
        return np.broadcast_to(grouped(v, groups).mean(axis=(2, 4), keepdims=True), (J, I, S, groups, D)).reshape(x.shape)

    dx = r * (h - over_group(h) - xh * over_group(h * xh))
    # errors of xh, of z and through the slope's derivative (at most 1/2) of dz
    e_xh = K * (np.abs(xh) + np.abs(x) * r * 2.0 ** -6)
    e_z = np.abs(w) * e_xh + K * (np.abs(z) + np.abs(b))
    e_dz = np.abs(da) * (K + (0.5 * e_z if kind == ACT_SILU else 0))
    e_h = np.abs(w) * e_dz + K * np.abs(h)
    s2 = over_group(np.abs(h * xh))
    bound = r * (e_h + over_group(e_h) + K * over_group(np.abs(h)) + np.abs(xh) * (over_group(e_h * np.abs(xh) + np.abs(h) * e_xh) + K * s2) +
                 e_xh * s2 + K * np.abs(h)) + 1e-37
    dweight, dbias = (dz * xh).sum(axis=(1, 2)), dz.sum(axis=(1, 2))
    b_w = (e_dz * np.abs(xh) + np.abs(dz) * e_xh + K * np.abs(dz * xh)).sum(axis=(1, 2)) + 1e-37
    b_b = (e_dz + K * np.abs(dz)).sum(axis=(1, 2)) + 1e-37
    return (dx, dweight, dbias), (bound, b_w, b_b)
