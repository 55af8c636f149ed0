"""The work that the products and the step of learners are measured on: matrix products with bias, activation and residual in their
epilogue, for all learners at once, with the gradients; and AdamW steps over the parameters of all learners.

A case is a dict of plain values.  ``kind`` selects the operator:

  product    x [sets][rows][inputs], weight [sets][outputs][inputs], fp32 bias [sets][outputs]:
             y = residual + act(x W^T + b), with ``keep`` also z = x W^T + b itself, as a training step wants it.
             ``turned``: the weights lie as [inputs][outputs]; ``wide`` > 0: x is the first columns of rows that long
  gradient   from dz, the gradient of z: dx = dz W (times the slope of ``act`` at the pre-activation that x came from),
             dW = dz^T x and db = sum of dz's rows in fp32; ``inner`` False: a first layer, without dx
  step       one AdamW step of ``learners`` nets whose parameters (``dims``: an MLP's weights and biases, or with ``blocks`` > 0 a net
             of normalised residual blocks) lie in rows of a matrix of replicas; ``bits`` 32 or 8 per value of a state,
             ``copy``: a bf16 copy of the parameters is written too
"""
import math

import numpy as np
import torch

own = False

_MOST_FLOPS = 2 * 8192 * 4096 * 16384      # of the largest case
_MOST_BYTES = 1 << 30
_MOST_PARAMS = 80_000_000
_BLOCK = 256                               # values of an 8-bit state that share a scale
_BORDER = 1.7320507764816284               # where the scale doubles (sqrt(3) in fp32: no sum of a few e4m3 and bf16 values, times beta, lies there)


def _product(sets, rows, inputs, outputs, bf16, act, residual=False, keep=False, turned=False, wide=0):
    return {"kind": "product", "sets": sets, "rows": rows, "inputs": inputs, "outputs": outputs, "bf16": bool(bf16), "act": act,
            "residual": bool(residual), "keep": bool(keep), "turned": bool(turned), "wide": wide}


def _gradient(sets, rows, inputs, outputs, bf16, act, inner=True, turned=False, wide=0):
    return {"kind": "gradient", "sets": sets, "rows": rows, "inputs": inputs, "outputs": outputs, "bf16": bool(bf16),
            "act": act if inner else "none", "inner": bool(inner), "turned": bool(turned), "wide": wide}


def _step(learners, dims, bits, bf16, copy, blocks=0):
    return {"kind": "step", "learners": learners, "dims": dims, "blocks": blocks, "bits": bits, "bf16": bool(bf16), "copy": bool(copy)}


def listed():
    cases = [
        # an answer for one sample through a wide hidden layer: the weights' bytes and latency
        ("product_one_row", _product(1, 1, 4096, 4096, True, "silu")),
        # a handful of samples through the layer behind it
        ("product_few_rows", _product(1, 11, 4096, 4096, True, "none", residual=True)),
        # last layer of the learners on CIFAR-shaped data, in fp32: few outputs
        ("product_head", _product(16, 128, 1024, 10, False, "none")),
        # their hidden layer in training
        ("product_hidden", _product(16, 128, 1024, 1024, True, "relu", keep=True)),
        # odd sizes in fp32, weights as residual blocks hold them, x out of a wider tensor
        ("product_odd", _product(3, 1003, 997, 515, False, "silu", residual=True, keep=True, turned=True, wide=1030)),
        # wide layer of one large net in training: the matrix cores
        ("product_large", _product(1, 8192, 4096, 16384, True, "silu", keep=True)),
        # the hidden layer of the learners, backward
        ("gradient_hidden", _gradient(16, 128, 1024, 1024, True, "relu")),
        # a residual block's product in fp32, rows of many positions, few channels
        ("gradient_positions", _gradient(8, 32 * 256, 64, 64, False, "silu", turned=True)),
        # the large net, backward
        ("gradient_large", _gradient(1, 8192, 4096, 4096, True, "silu")),
        # learners of residual blocks: many small parameters
        ("step_blocks", _step(8, "27,64,10", 32, False, False, blocks=2)),
        # learners of the widest hidden layers, with the copy that their products read
        ("step_wide", _step(2, "4096,4096,4096,1000", 32, False, True)),
        # the same with states in 8 bits and gradients in bf16
        ("step_wide_8bit", _step(2, "4096,4096,4096,1000", 8, True, True)),
    ]
    return [dict(case, name=name) for name, case in cases]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """The same; half of them multiples of 8 (or of a larger power of two)."""
    n = _log(rng, lo, hi)
    if rng.random() < 0.5:
        unit = rng.choice((8, 32, 64, 256))
        n = min(hi, max(unit, n // unit * unit))
    return n


def _draw_product(rng):
    sets = 1 if rng.random() < 0.4 else _log(rng, 2, 16)
    rows = _log(rng, 1, 32) if rng.random() < 0.3 else _size(rng, 1, 16384)
    inputs, outputs = _size(rng, 8, 16384), _size(rng, 1, 16384)
    flops, values = 2 * sets * rows * inputs * outputs, sets * (rows * (inputs + 3 * outputs) + inputs * outputs)
    bf16, turned, back = rng.random() < 0.6, rng.random() < 0.3, rng.random() < 0.4
    if flops < 1 << 14 or flops > _MOST_FLOPS // (2 if back else 1) // (1 if bf16 else 8) or 4 * values > _MOST_BYTES:
        return None
    wide = inputs + _log(rng, 1, inputs) if rng.random() < 0.2 else 0
    if back:
        return _gradient(sets, rows, inputs, outputs, bf16, rng.choice(("none", "relu", "silu")), inner=rng.random() < 0.85, turned=turned, wide=wide)
    return _product(sets, rows, inputs, outputs, bf16, rng.choice(("none", "relu", "silu")), residual=rng.random() < 0.4, keep=rng.random() < 0.4,
                    turned=turned, wide=wide)


def _draw_step(rng):
    blocks = rng.randrange(1, 9) if rng.random() < 0.4 else 0
    dims = [_size(rng, 16, 4096) for _ in range(2 if blocks else rng.randrange(2, 5))] + [_log(rng, 2, 1000)]
    learners = _log(rng, 1, 16)
    case = _step(learners, ",".join(map(str, dims)), rng.choice((32, 32, 8)), rng.random() < 0.4, rng.random() < 0.5, blocks=blocks)
    return case if learners * sum(math.prod(s) for s in _shapes(case)) <= _MOST_PARAMS else None


def draw(rng):
    """One more case of the ranges above."""
    make = rng.choices((_draw_product, _draw_step), (5, 2))[0]
    while True:
        case = make(rng)
        if case is not None:
            return case


def _shapes(case):
    """Shapes of a learner's parameters."""
    d = [int(n) for n in case["dims"].split(",")]
    if not case["blocks"]:
        return [s for a, b in zip(d, d[1:]) for s in ((b, a), (b,))]
    c_in, c, classes = d
    shapes = [(c_in, c)]
    for _ in range(case["blocks"]):
        shapes += [(c,), (c,), (c, c)]
    return shapes + [(c,), (c,), (c, classes), (classes,)]


# ---- inputs ------------------------------------------------------------------------------------------------------

_OPTIONS = {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01}


def _normal(gen, *shape, scale=1.0, dtype=torch.float32):
    return torch.empty(*shape, device="cuda").normal_(0, scale, generator=gen).to(dtype)


def _prepare_product(case, gen, state):
    J, M, K, N = (case[k] for k in ("sets", "rows", "inputs", "outputs"))
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    state["x"] = _normal(gen, J, M, case["wide"] or K, dtype=dtype)[..., :K]
    # a learner's weights and biases lie in its row of the replicas (of their bf16 copies)
    row = (N * K + N + 7) // 8 * 8
    rows = _normal(gen, J, row, scale=K ** -0.5, dtype=dtype)
    w = rows[:, :N * K]
    state["weight"] = w.view(J, K, N).transpose(1, 2) if case["turned"] else w.view(J, N, K)
    if case["kind"] == "product":
        state["bias"] = _normal(gen, J, row, scale=0.1)[:, N * K:N * K + N]
        state["residual_y"] = _normal(gen, J, M, N, dtype=dtype) if case["residual"] else None
    else:
        state["dz"] = _normal(gen, J, M, N, scale=1e-2, dtype=dtype)
        state["pre"] = _normal(gen, J, M, K, dtype=dtype) if case["act"] != "none" else None
    return state


def _prepare_step(case, gen, state):
    P, shapes = case["learners"], _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    n = (sum(sizes) + 7) // 8 * 8
    state["replicas"], state["copies"] = torch.zeros(P, n, device="cuda"), None
    if case["copy"]:
        state["copies"] = torch.zeros(P, n, dtype=torch.bfloat16, device="cuda")
    for k in ("params", "grads", "states", "copy_of"):
        state[k] = []
    eight = case["bits"] == 8
    blocks = [(size + _BLOCK - 1) // _BLOCK for size in sizes]
    kept = {"m": (torch.float8_e4m3fn if eight else torch.float32, sizes), "v": (torch.float8_e4m3fn if eight else torch.float32, sizes)}
    if eight:
        kept.update({"m_scale": (torch.float32, blocks), "v_scale": (torch.float32, blocks)})
    state["kept"] = {k: torch.zeros(P * sum(each), dtype=t, device="cuda") for k, (t, each) in kept.items()}
    at = {k: 0 for k in ("params", *kept)}
    for shape, size in zip(shapes, sizes):
        p = state["replicas"][:, at["params"]:at["params"] + size].view(P, *shape)
        if len(shape) > 1:
            p.normal_(0, shape[-1] ** -0.5, generator=gen)
        state["params"].append(p)
        state["copy_of"].append(state["copies"][:, at["params"]:at["params"] + size].view(P, *shape) if case["copy"] else None)
        at["params"] += size
        # gradients of different sizes from row to row, and the moments that a hundred such left
        spread = torch.exp(_normal(gen, P, *shape[:-1], 1)) * 1e-3
        grad = _normal(gen, P, *shape) * spread
        m = (0.3 * _normal(gen, P, *shape)) * spread
        v = (0.1 * (1 + 0.2 * _normal(gen, P, *shape)) * spread).square()
        state["grads"].append(grad.to(torch.bfloat16 if case["bf16"] else torch.float32))
        views = {}
        for k, (_, each) in kept.items():
            length = P * each[len(state["params"]) - 1]
            views[k] = state["kept"][k][at[k]:at[k] + length].view(P, *(shape if k in "mv" else (-1,)))
            at[k] += length
        if eight:
            none = torch.full((P, size), 0.5, device="cuda")
            for k, value in (("m", m.view(P, size)), ("v", v.view(P, size).sqrt())):
                codes, scale = _coded(value, none if k == "v" else None)
                views[k].copy_(codes.view(views[k].shape))
                views[k + "_scale"].copy_(scale)
        else:
            views["m"].copy_(m)
            views["v"].copy_(v)
        state["states"].append(tuple(views[k] for k in kept))
    state["step"] = 100
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case, seed=seed * 0x9E3779B1 % (1 << 63))
    return _prepare_step(case, gen, state) if case["kind"] == "step" else _prepare_product(case, gen, state)


# ---- plain forms -------------------------------------------------------------------------------------------------

def _plain_product(s):
    x, dtype = s["x"], s["x"].dtype
    z = torch.matmul(x.float(), s["weight"].float().transpose(1, 2)) + s["bias"][:, None]
    y = z
    if s["act"] == "relu":
        y = z.clamp(min=0)
    elif s["act"] == "silu":
        y = z / (1 + torch.exp(-z))
    if s["residual"]:
        y = y + s["residual_y"].float()
    return {"y": y.to(dtype), "pre": z.to(dtype)} if s["keep"] else {"y": y.to(dtype)}


def _plain_gradient(s):
    dz, out = s["dz"].float(), {}
    if s["inner"]:
        dx = torch.matmul(dz, s["weight"].float())
        if s["act"] == "relu":
            dx = torch.where(s["pre"] > 0, dx, 0.0)
        elif s["act"] == "silu":
            z = s["pre"].float()
            g = 1 / (1 + torch.exp(-z))
            dx = dx * (g * (1 + z * (1 - g)))
        out["dx"] = dx.to(s["dz"].dtype)
    out["dweight"] = torch.matmul(dz.transpose(1, 2), s["x"].float())
    out["dbias"] = dz.sum(1)
    return out


def _shifted(z, n):
    """Logical right shift of 64-bit words."""
    return (z >> n) & ((1 << (64 - n)) - 1)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _draws(shape, seed, site):
    """Element e's draw from [0, 1): the 16 bits, the (e mod 4)-th, of output number 1 + site 2^40 + e / 4 of SplitMix64, and a half."""
    n = math.prod(shape)
    z = (torch.arange(1, (n + 3) // 4 + 1, dtype=torch.int64, device="cuda") + (site << 40)) * _signed(0x9E3779B97F4A7C15) + _signed(seed)
    z = (z ^ _shifted(z, 30)) * _signed(0xBF58476D1CE4E5B9)
    z = (z ^ _shifted(z, 27)) * _signed(0x94D049BB133111EB)
    z = z ^ _shifted(z, 31)
    bits = ((z[:, None] >> torch.arange(0, 64, 16, device="cuda")) & 0xFFFF).view(-1)[:n]
    return ((2 * bits + 1).float() * 2.0 ** -17).view(shape)


def _coded(value, draws):
    """[rows][n] in fp32 as e4m3 values and a scale, a power of two, for every 256 of a row: the largest of them is 128 to 256
    times _BORDER scales.  To nearest, or with draws (values that are not negative) up where the draw plus the remainder reaches one, never from above zero to zero."""
    rows, n = value.shape
    pad = torch.zeros(rows, -n % _BLOCK, device=value.device)
    v = torch.cat((value, pad), 1).view(rows, -1, _BLOCK)
    most = v.abs().amax(2)
    part, exponent = torch.frexp(most)                               # most = part 2^exponent, part in [1/2, 1)
    exponent = torch.where(most > 0, exponent - 9 + (part >= 0.5 * _BORDER), -126)
    scale = torch.ldexp(torch.ones_like(most), exponent.clamp(min=-126))
    q = v / scale[..., None]
    if draws is None:
        q = q.to(torch.float8_e4m3fn)
    else:
        d = torch.cat((draws, pad), 1).view_as(v)
        unit = torch.ldexp(torch.ones_like(q), torch.frexp(q)[1].clamp(min=-5) - 4)     # distance of e4m3's values here
        up = torch.floor(q / unit)
        up = (up + ((q / unit - up) + d >= 1)) * unit
        q = torch.where(q > 0, up.clamp(min=2.0 ** -9), 0.0).to(torch.float8_e4m3fn)
    return q.view(rows, -1)[:, :n], scale


def _plain_step(s):
    P, o, t, eight = s["learners"], _OPTIONS, s["step"], s["bits"] == 8
    c1, c2 = 1 - o["beta1"] ** t, 1 - o["beta2"] ** t
    for i, (p, grad, kept, copy) in enumerate(zip(s["params"], s["grads"], s["states"], s["copy_of"])):
        g = grad.float()
        if eight:
            across = [kept[k].repeat_interleave(_BLOCK, 1)[:, :g[0].numel()].view(g.shape) for k in (2, 3)]
            m, root = kept[0].float() * across[0], kept[1].float() * across[1]
            v = root * root
        else:
            m, v = kept[:2]
        m = m * o["beta1"] + g * (1 - o["beta1"])
        v = v * o["beta2"] + (g * g) * (1 - o["beta2"])
        root = v.sqrt()
        new = p * (1 - o["lr"] * o["weight_decay"]) - (o["lr"] / c1) * (m / (root / math.sqrt(c2) + o["eps"]))
        p.copy_(new)
        if copy is not None:                                         # to nearest, ties away from zero
            copy.copy_((((new.contiguous().view(torch.int32) + 0x8000) >> 16) << 16).view(torch.float32))
        if eight:
            draws = _draws((P, g[0].numel()), s["seed"] + t, i)
            for k, value, d in ((0, m, None), (1, root, draws)):
                codes, scale = _coded(value.reshape(P, -1), d)
                kept[k].copy_(codes.view(kept[k].shape))
                kept[2 + k].copy_(scale)
        else:
            kept[0].copy_(m)
            kept[1].copy_(v)
    return _state_of(s)


def _state_of(s):
    out = dict(s["kept"], params=s["replicas"])
    if s["copies"] is not None:
        out["copies"] = s["copies"]
    s["step"] += 1
    return out


# ---- the calls of a user's program -------------------------------------------------------------------------------

def _own(s):
    from paper_2110_00625_amd import kavg
    if s["kind"] == "step":
        if "plan" not in s:                                          # (a program makes it once, with its states)
            s["plan"] = kavg.AdamW(s["params"], states=s["states"], copies=s["copy_of"] if s["copy"] else None)
        s["plan"].step(s["grads"], s["step"], seed=s["seed"], **_OPTIONS)
        return _state_of(s)
    act = {"none": kavg.KAVG_ACT_NONE, "relu": kavg.KAVG_ACT_RELU, "silu": kavg.KAVG_ACT_SILU}[s["act"]]
    if s["kind"] == "product":
        out = kavg.kavg_linear(s["x"], s["weight"], s["bias"], activation=act, residual=s["residual_y"], pre=s["keep"])
        return {"y": out[0], "pre": out[1]} if s["keep"] else {"y": out}
    dx, dweight, dbias = kavg.kavg_linear_backward(s["dz"], s["x"], s["weight"], activation=act, pre=s["pre"], out=None if s["inner"] else False)
    return {"dx": dx, "dweight": dweight, "dbias": dbias} if s["inner"] else {"dweight": dweight, "dbias": dbias}


def run(state):
    if own:
        return _own(state)
    return {"product": _plain_product, "gradient": _plain_gradient, "step": _plain_step}[state["kind"]](state)


def work(case):
    if case["kind"] == "step":
        sizes = [math.prod(s) for s in _shapes(case)]
        n, blocks = case["learners"] * sum(sizes), case["learners"] * sum((s + _BLOCK - 1) // _BLOCK for s in sizes)
        each = 8 + (2 if case["bf16"] else 4) + (16 if case["bits"] == 32 else 4) + (2 if case["copy"] else 0)
        return {"bytes": n * each + (16 * blocks if case["bits"] == 8 else 0), "flops": 15 * n}
    J, M, K, N = (case[k] for k in ("sets", "rows", "inputs", "outputs"))
    e = 2 if case["bf16"] else 4
    if case["kind"] == "product":
        outputs = 1 + case["keep"] + case["residual"]
        return {"bytes": J * (e * (M * K + N * K + outputs * M * N) + 4 * N), "flops": J * M * N * (2 * K + 6)}
    inner = e * (M * K * (2 if case["act"] != "none" else 1) + N * K) if case["inner"] else 0
    return {"bytes": J * (e * (M * N + M * K) + inner + 4 * (N * K + N)), "flops": 2 * J * M * N * K * (2 if case["inner"] else 1)}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------

def _exact_product(s):
    """Learner by learner, some rows at once; sigmoid by tanh."""
    parts = {"y": [], "pre": []}
    for j in range(s["sets"]):
        w, b = s["weight"][j].double(), s["bias"][j].double()
        for r in range(0, s["rows"], 2048):
            z = torch.addmm(b, s["x"][j, r:r + 2048].double(), w.t())
            y = {"none": lambda t: t, "relu": torch.relu, "silu": lambda t: t * (0.5 + 0.5 * torch.tanh(0.5 * t))}[s["act"]](z)
            parts["y"].append(y + s["residual_y"][j, r:r + 2048].double() if s["residual"] else y)
            parts["pre"].append(z if s["keep"] else None)
    shape = (s["sets"], s["rows"], s["outputs"])
    return {k: torch.cat(parts[k]).view(shape) for k in (("y", "pre") if s["keep"] else ("y",))}


def _exact_gradient(s):
    parts = {"dx": [], "dweight": [], "dbias": []}
    for j in range(s["sets"]):
        w = s["weight"][j].double()
        dw, db = torch.zeros_like(w), torch.zeros(s["outputs"], dtype=torch.float64, device="cuda")
        for r in range(0, s["rows"], 2048):
            dz, x = s["dz"][j, r:r + 2048].double(), s["x"][j, r:r + 2048].double()
            dw = torch.addmm(dw, dz.t(), x)
            db += dz.sum(0)
            if s["inner"]:
                dx = dz @ w
                if s["act"] != "none":
                    z = s["pre"][j, r:r + 2048].double()
                    sig = 0.5 + 0.5 * torch.tanh(0.5 * z)
                    dx = dx * ((z > 0).double() if s["act"] == "relu" else sig + z * sig * (1 - sig))
                parts["dx"].append(dx)
        parts["dweight"].append(dw)
        parts["dbias"].append(db)
    out = {"dweight": torch.stack(parts["dweight"]), "dbias": torch.stack(parts["dbias"])}
    return dict(out, dx=torch.cat(parts["dx"]).view(s["sets"], s["rows"], s["inputs"])) if s["inner"] else out


def _words(n, seed, site):
    """The draws in numpy's unsigned words and their 16-bit quarters."""
    z = np.arange(1, (n + 3) // 4 + 1, dtype=np.uint64) + np.uint64(site << 40)
    with np.errstate(over="ignore"):
        z = np.uint64(seed) + z * np.uint64(0x9E3779B97F4A7C15)
        for shift, factor in ((30, 0xBF58476D1CE4E5B9), (27, 0x94D049BB133111EB)):
            z ^= z >> np.uint64(shift)
            z *= np.uint64(factor)
        z ^= z >> np.uint64(31)
    return torch.from_numpy((z.astype("<u8").view("<u2")[:n].astype(np.float64) + 0.5) / 65536).cuda()


def _grid(v, draws):
    """[n] in 64 bits as (multiples of e4m3's distances, scale per block): by logarithms; to nearest, ties to even, where draws is None."""
    n = v.numel()
    most = torch.zeros((n + _BLOCK - 1) // _BLOCK * _BLOCK, dtype=torch.float64, device="cuda")
    most[:n] = v.abs()
    most = most.view(-1, _BLOCK).max(1).values
    scale = torch.where(most > 0, 2.0 ** (torch.floor(torch.log2(most.clamp(min=1e-300) / _BORDER)) - 7), 0.0).clamp(min=2.0 ** -126)
    q = v / scale[torch.arange(n, device="cuda") // _BLOCK]
    unit = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
    k = torch.round(q / unit) if draws is None else torch.floor(q / unit + draws)
    if draws is not None:
        k = torch.where((q > 0) & (k == 0), 1.0, k)
    return k * unit, scale


def _exact_step(s):
    o, t, eight, P = _OPTIONS, s["step"], s["bits"] == 8, s["learners"]
    lr, b1, b2 = o["lr"], o["beta1"], o["beta2"]
    parts = {k: [] for k in s["kept"]}
    whole = torch.zeros_like(s["replicas"], dtype=torch.float64)
    at = 0
    for i, (p, grad, kept) in enumerate(zip(s["params"], s["grads"], s["states"])):
        n = p[0].numel()
        draws = _words(P * n, (s["seed"] + t) & ((1 << 64) - 1), i).view(P, n) if eight else None
        for j in range(P):
            g, w = grad[j].double().flatten(), p[j].double().flatten()
            m, v = kept[0][j].double().flatten(), kept[1][j].double().flatten()
            if eight:
                block = torch.arange(n, device="cuda") // _BLOCK
                m, v = m * kept[2][j].double()[block], (v * kept[3][j].double()[block]).square()
            m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g.square()
            whole[j, at:at + n] = w - lr * o["weight_decay"] * w - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + o["eps"])
            if eight:
                m, m_scale = _grid(m, None)
                v, v_scale = _grid(v.sqrt(), draws[j])
                parts["m_scale"].append(m_scale)
                parts["v_scale"].append(v_scale)
            parts["m"].append(m)
            parts["v"].append(v)
        at += n
    out = {k: torch.cat(v) for k, v in parts.items()}
    out["params"] = whole
    if s["copies"] is not None:
        out["copies"] = whole
    return out


def exact(case, seed):
    return {"product": _exact_product, "gradient": _exact_gradient, "step": _exact_step}[case["kind"]](prepare(case, seed))
