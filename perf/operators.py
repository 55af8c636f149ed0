"""The work the normalisation and regularisation operators are measured on: group norm with an activation (and dropout
as its epilogue) on channels-last images of several learners, and dropout of the rows of a layer's activations.

A case is a dict of plain values.  ``kind`` selects the operator, ``backward`` its direction:

  norm   x [sets][images][positions][channels], parameters [sets][channels], ``groups`` groups of channels;
         ``act`` "none", "relu" or "silu"; ``drop`` > 0 drops activations behind it; ``wide`` > 0: x is the first
         ``channels`` channels of rows of ``wide`` values, as behind a concatenation
  drop   x [rows][cols], with ``residual`` the sum of a residual and the dropped x; ``wide`` as above

ReLU is measured forward only: its derivative jumps at zero, so two right backward passes may differ by a whole element
where a pre-activation lies within a rounding of zero.
"""
import math

import numpy as np
import torch

own = False

_EPS = 1e-5
_MOST = 16 * 64 * 1024 * 128          # elements of the largest case


def _norm(sets, images, positions, channels, groups, bf16, act, drop=0.0, backward=False, stats=True, wide=0):
    return {"kind": "norm", "sets": sets, "images": images, "positions": positions, "channels": channels,
            "groups": groups, "bf16": bool(bf16), "act": act, "drop": drop, "backward": backward,
            "stats": bool(stats or backward), "wide": wide}


def _drop(rows, cols, bf16, drop, residual=False, backward=False, wide=0):
    return {"kind": "drop", "rows": rows, "cols": cols, "bf16": bool(bf16), "drop": drop,
            "residual": bool(residual and not backward), "backward": backward, "wide": wide}


def listed():
    cases = [
        # an answer for one small image: nothing but latency
        ("norm_one_image", _norm(1, 1, 64, 64, 8, True, "relu", stats=False)),
        # vectors rather than images: the rows of a 1024-wide hidden layer, one position each
        ("norm_vectors", _norm(1, 1000, 1, 1024, 16, False, "silu")),
        # last convolution of the learners on CIFAR-shaped images, a whole minibatch of each
        ("norm_cifar", _norm(16, 64, 32 * 32, 128, 8, True, "relu", drop=0.1)),
        # the convolution before it, backward
        ("norm_cifar_backward", _norm(16, 64, 32 * 32, 64, 8, True, "silu", drop=0.1, backward=True)),
        # images of another width, channels that fill no line, in fp32
        ("norm_28_backward", _norm(8, 32, 28 * 28, 40, 5, False, "silu", backward=True)),
        # deep and small images, read out of a wider tensor
        ("norm_deep_backward", _norm(1, 256, 16, 512, 32, True, "silu", drop=0.2, backward=True, wide=768)),
        # few large images: a group's positions exceed what one compute unit holds
        ("norm_large_images", _norm(1, 2, 256 * 256, 128, 32, True, "silu")),
        # the same in training, at an odd size, ten channels to a group
        ("norm_large_images_backward", _norm(1, 3, 127 * 129, 320, 32, True, "silu", backward=True)),
        # hidden layer of the sweep's learners: 48 minibatches of 4, again latency
        ("drop_small", _drop(48 * 4, 256, False, 0.5)),
        # hidden layer of the largest model, all learners' minibatches, added to a residual
        ("drop_residual", _drop(8 * 256, 4096, True, 0.1, residual=True)),
        # odd rows of an odd length
        ("drop_odd_backward", _drop(4999, 1001, False, 0.2, backward=True)),
        # activations of all positions of the CIFAR-shaped learners
        ("drop_images_backward", _drop(16 * 64 * 32 * 32, 64, True, 0.1, backward=True)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_norm(rng):
    backward = rng.random() < 0.5
    if rng.random() < 0.15:
        positions = 1
    else:
        h = _log(rng, 3, 256)
        positions = h * (h if rng.random() < 0.5 else _log(rng, 3, 256))
    per, groups = _log(rng, 1, 64), _log(rng, 1, 64)
    if rng.random() < 0.5:
        per, groups = 1 << int(math.log2(per)), 1 << int(math.log2(groups))
    sets, images, channels = _log(rng, 1, 16), _log(rng, 1, 512), per * groups
    n = sets * images * positions * channels
    if channels < 4 or channels > 2048 or positions * per < 16 or n > (_MOST // 2 if backward else _MOST):
        return None
    wide = channels + _log(rng, 1, channels) if rng.random() < 0.2 and n <= _MOST // 4 else 0
    return _norm(sets, images, positions, channels, groups, rng.random() < 0.6,
                 rng.choice(("none", "silu") if backward else ("none", "relu", "silu", "silu")),
                 drop=rng.choice((0.0, 0.0, 0.1, 0.25, 0.5)), backward=backward, stats=rng.random() < 0.7, wide=wide)


def _draw_drop(rng):
    rows, cols = _log(rng, 1, 1 << 20), _log(rng, 1, 8192)
    if rng.random() < 0.5:
        cols = (cols + 7) // 8 * 8
    if rows * cols < 64 or rows * cols > _MOST // 2:
        return None
    wide = cols + _log(rng, 1, cols) if rng.random() < 0.2 and rows * cols <= _MOST // 4 else 0
    backward = rng.random() < 0.5
    return _drop(rows, cols, rng.random() < 0.6, rng.choice((0.05, 0.1, 0.25, 0.5, 0.9)), residual=rng.random() < 0.5,
                 backward=backward, wide=wide)


def draw(rng):
    """One more case of the ranges above."""
    make = rng.choices((_draw_norm, _draw_drop), (2, 1))[0]
    while True:
        case = make(rng)
        if case is not None:
            return case


def _tensor(shape, wide, dtype, gen):
    """N(0, 1) values; with `wide`, the first columns of rows that long."""
    at = torch.empty(*shape[:-1], wide or shape[-1], dtype=dtype, device="cuda")
    return at.normal_(generator=gen)[..., :shape[-1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    state = dict(case, seed=seed * 0x9E3779B1 % (1 << 63), site=seed % 97)
    if case["kind"] == "drop":
        shape = (case["rows"], case["cols"])
        state["x"] = _tensor(shape, case["wide"], dtype, gen)
        if case["residual"]:
            state["residual_x"] = _tensor(shape, 0, dtype, gen)
        return state
    J, I, S, C, G = (case[k] for k in ("sets", "images", "positions", "channels", "groups"))
    # what a convolution leaves: every channel with an offset and a spread of its own
    x = _tensor((J, I, S, C), case["wide"], dtype, gen)
    x *= torch.rand(J, 1, 1, C, generator=gen, device="cuda").to(dtype) + 0.5
    x += torch.randn(J, 1, 1, C, generator=gen, device="cuda").to(dtype) * 0.5 + 0.25
    state["x"] = x
    state["weight"] = 1 + 0.2 * torch.randn(J, C, generator=gen, device="cuda")
    state["bias"] = 0.2 * torch.randn(J, C, generator=gen, device="cuda")
    if case["backward"]:
        # the statistics that the forward pass left
        rows = x.reshape(J * I, S, C).split(max(1, (1 << 26) // (S * C)))
        both = [torch.var_mean(r.double().view(-1, S, G, C // G), (1, 3), correction=0) for r in rows]
        state["mean"] = torch.cat([m for _, m in both]).float().view(J, I, G)
        state["rstd"] = torch.cat([(v + _EPS).rsqrt() for v, _ in both]).float().view(J, I, G)
        state["dy"] = _tensor((J, I, S, C), 0, dtype, gen)
    return state


# ---- plain forms -------------------------------------------------------------------------------------------------

def _shifted(z, n):
    """Logical right shift of 64-bit words."""
    return (z >> n) & ((1 << (64 - n)) - 1)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _kept(n, drop, seed, site):
    """Element e goes by 16 bits, the (e mod 4)-th, of output number 1 + site 2^40 + e / 4 of SplitMix64."""
    count = torch.arange(1, (n + 3) // 4 + 1, dtype=torch.int64, device="cuda") + (site << 40)
    z = count * _signed(0x9E3779B97F4A7C15) + _signed(seed)
    z = (z ^ _shifted(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shifted(z, 27)) * _signed(0x94D049BB133111EB)
    z = z ^ _shifted(z, 31)
    bits = (z[:, None] >> torch.arange(0, 64, 16, device="cuda")) & 0xFFFF
    return bits.view(-1)[:n] >= int(drop * 65536 + 0.5)


def _scale(drop):
    gone = int(drop * 65536 + 0.5)
    return 65536.0 / (65536 - gone) if gone < 65536 else 0.0


def _dropped(x, drop, seed, site):
    """fp32 x with its dropped elements zero and the others scaled."""
    return torch.where(_kept(x.numel(), drop, seed, site).view(x.shape), x * _scale(drop), 0.0)


def _plain_drop(s):
    y = _dropped(s["x"].float(), s["drop"], s["seed"], s["site"])
    if s["residual"]:
        y = y + s["residual_x"].float()
    return y.to(s["x"].dtype)


def _plain_norm(s):
    x, G = s["x"], s["groups"]
    J, I, S, C = x.shape
    xg = x.float().reshape(J, I, S, G, C // G)
    mean = xg.mean((2, 4), keepdim=True)
    centred = xg - mean
    rstd = ((centred * centred).mean((2, 4), keepdim=True) + _EPS) ** -0.5
    y = (centred * rstd).view(J, I, S, C) * s["weight"].view(J, 1, 1, C) + s["bias"].view(J, 1, 1, C)
    if s["act"] == "relu":
        y = y.clamp(min=0)
    elif s["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    if s["drop"]:
        y = _dropped(y, s["drop"], s["seed"], s["site"])
    y = y.to(x.dtype)
    return {"y": y, "mean": mean.view(J, I, G), "rstd": rstd.view(J, I, G)} if s["stats"] else {"y": y}


def _plain_norm_backward(s):
    x, G = s["x"], s["groups"]
    J, I, S, C = x.shape
    D = C // G
    w = s["weight"].view(J, 1, 1, C)
    rstd = s["rstd"].view(J, I, 1, G, 1)
    xh = ((x.float().reshape(J, I, S, G, D) - s["mean"].view(J, I, 1, G, 1)) * rstd).view(J, I, S, C)
    dz = s["dy"].float()
    if s["drop"]:
        dz = _dropped(dz, s["drop"], s["seed"], s["site"])
    if s["act"] == "silu":
        z = xh * w + s["bias"].view(J, 1, 1, C)
        g = 1 / (1 + torch.exp(-z))
        dz = dz * (g * (1 + z * (1 - g)))
    dxh = dz * xh
    h, hx = (dz * w).view(J, I, S, G, D), (dxh * w).view(J, I, S, G, D)
    dx = h - h.mean((2, 4), keepdim=True) - xh.view(J, I, S, G, D) * hx.mean((2, 4), keepdim=True)
    return {"dx": (dx * rstd).view(J, I, S, C).to(x.dtype), "dweight": dxh.sum((1, 2)), "dbias": dz.sum((1, 2))}


# ---- the calls of a user's program -------------------------------------------------------------------------------

def _own(s):
    from paper_2110_00625_amd import kavg
    if s["kind"] == "drop":
        if s["backward"]:
            return kavg.kavg_dropout_backward(s["x"], s["drop"], s["seed"], site=s["site"])
        return kavg.kavg_dropout(s["x"], s["drop"], s["seed"], site=s["site"],
                                 residual=s["residual_x"] if s["residual"] else None)
    act = {"none": kavg.KAVG_ACT_NONE, "relu": kavg.KAVG_ACT_RELU, "silu": kavg.KAVG_ACT_SILU}[s["act"]]
    if s["backward"]:
        dx, dweight, dbias = kavg.kavg_group_norm_backward(
            s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], s["bias"], s["groups"], activation=act,
            drop=s["drop"], seed=s["seed"], site=s["site"])
        return {"dx": dx, "dweight": dweight, "dbias": dbias}
    out = kavg.kavg_group_norm(s["x"], s["weight"], s["bias"], s["groups"], eps=_EPS, activation=act, drop=s["drop"],
                               seed=s["seed"], site=s["site"], stats=s["stats"])
    return dict(zip(("y", "mean", "rstd"), out)) if s["stats"] else {"y": out}


def run(state):
    if own:
        return _own(state)
    if state["kind"] == "drop":
        return _plain_drop(state)           # the gradient of dropout is dropout of the gradient
    return _plain_norm_backward(state) if state["backward"] else _plain_norm(state)


def work(case):
    e = 2 if case["bf16"] else 4
    if case["kind"] == "drop":
        n = case["rows"] * case["cols"]
        return {"bytes": (3 if case["residual"] else 2) * n * e, "flops": (2 if case["residual"] else 1) * n}
    J, I, S, C, G = (case[k] for k in ("sets", "images", "positions", "channels", "groups"))
    n = J * I * S * C
    act = {"none": 0, "relu": 1, "silu": 4}[case["act"]]
    if case["backward"]:
        # x, dy, dx; both statistics, both parameters and their gradients
        return {"bytes": 3 * n * e + 8 * J * I * G + 16 * J * C, "flops": (14 + 2 * act) * n}
    return {"bytes": 2 * n * e + (8 * J * I * G if case["stats"] else 0) + 8 * J * C, "flops": (8 + act) * n}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------

def _keep_factors(first, n, drop, seed, site):
    """0 or the scale for n elements from the first-th on, from numpy's unsigned words and their 16-bit quarters."""
    c = np.arange(first // 4, (first + n - 1) // 4 + 1, dtype=np.uint64) + np.uint64((site << 40) + 1)
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + c * np.uint64(0x9E3779B97F4A7C15)
        for shift, factor in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB)):
            z ^= z >> np.uint64(shift)
            z *= np.uint64(factor)
        z ^= z >> np.uint64(31)
    gone = math.floor(drop * 65536 + 0.5)
    quarters = z.astype("<u8").view("<u2")[first % 4:first % 4 + n]
    return torch.from_numpy(quarters >= gone).cuda().double() * (65536.0 / (65536 - gone))


def _exact_norm(s):
    """Image by image; sums of a group's values and squares of their distances from the mean."""
    x, G = s["x"], s["groups"]
    J, I, S, C = x.shape
    D = C // G
    w, b = s["weight"].double(), s["bias"].double()
    at_once = max(1, (1 << 24) // (S * C))
    parts = {k: [] for k in (("dx", "dweight", "dbias") if s["backward"] else ("y", "mean", "rstd"))}
    for j in range(J):
        dw = torch.zeros(C, dtype=torch.float64, device="cuda")
        db = torch.zeros_like(dw)
        for i in range(0, I, at_once):
            v = x[j, i:i + at_once].double().permute(0, 2, 1).reshape(-1, G, D * S)       # [images][groups][values]
            k = v.shape[0]
            if s["backward"]:
                mean = s["mean"][j, i:i + k].double()[..., None]
                rstd = s["rstd"][j, i:i + k].double()[..., None]
            else:
                mean = v.sum(-1, keepdim=True) / (D * S)
                rstd = ((v - mean).square().sum(-1, keepdim=True) / (D * S) + _EPS).sqrt().reciprocal()
            xh = ((v - mean) * rstd).view(k, C, S)
            z = w[j, :, None] * xh + b[j, :, None]
            factor = torch.ones((), dtype=torch.float64, device="cuda")
            if s["drop"]:
                factor = _keep_factors((j * I + i) * S * C, k * S * C, s["drop"], s["seed"], s["site"])
                factor = factor.view(k, S, C).permute(0, 2, 1)
            if not s["backward"]:
                a = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * torch.sigmoid(t)}[s["act"]](z)
                parts["y"].append((a * factor).permute(0, 2, 1))
                parts["mean"].append(mean[..., 0])
                parts["rstd"].append(rstd[..., 0])
                continue
            dz = s["dy"][j, i:i + k].double().permute(0, 2, 1) * factor
            if s["act"] == "silu":
                sig = torch.sigmoid(z)
                dz = dz * (sig + z * sig * torch.sigmoid(-z))
            db += dz.sum((0, 2))
            dw += (dz * xh).sum((0, 2))
            h, xh = (dz * w[j, :, None]).reshape(k, G, D * S), xh.reshape(k, G, D * S)
            dv = rstd * (h - h.sum(-1, keepdim=True) / (D * S) - xh * ((h * xh).sum(-1, keepdim=True) / (D * S)))
            parts["dx"].append(dv.reshape(k, C, S).permute(0, 2, 1))
        if s["backward"]:
            parts["dweight"].append(dw)
            parts["dbias"].append(db)
    shapes = {"y": (J, I, S, C), "dx": (J, I, S, C), "mean": (J, I, G), "rstd": (J, I, G)}
    out = {k: torch.cat(v).view(shapes[k]) if k in shapes else torch.stack(v) for k, v in parts.items()}
    return out if s["stats"] else {"y": out["y"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    rows, cols = case["rows"], case["cols"]
    y = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 24) // cols)
    for r in range(0, rows, step):
        k = min(step, rows - r)
        factors = _keep_factors(r * cols, k * cols, case["drop"], s["seed"], s["site"])
        y[r:r + k] = s["x"][r:r + k].double() * factors.view(k, cols)
    return y + s["residual_x"].double() if case["residual"] else y
