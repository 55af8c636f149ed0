"""kavg_group_norm and its backward pass against the 64-bit forms of layers_reference.py, within the bounds derived there."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import layers_reference as R

pytestmark = pytest.mark.gpu

DTYPES = (torch.float32, torch.bfloat16)
# sets, images, positions, channels, groups
SHAPES = [
    (1, 1, 1, 1, 1), (1, 1, 1, 4, 2), (1, 5, 1, 1024, 16), (3, 2, 1, 40, 40), (1, 1, 2, 8, 1), (2, 3, 7, 12, 3), (1, 1, 64, 64, 8),
    (3, 2, 33, 40, 5), (2, 2, 49, 91, 7), (1, 3, 5, 23, 23), (1, 2, 30, 7, 1), (1, 2, 17, 2040, 8), (1, 1, 9, 2047, 23), (1, 2, 300, 320, 32),
    (2, 1, 1100, 128, 32), (1, 1, 4097, 8, 2), (1, 2, 1024, 64, 8), (4, 33, 16, 32, 4), (1, 300, 3, 10, 5), (1, 1, 2500, 50, 5),
    (2, 1, 16383, 16, 4), (1, 1, 20000, 33, 3), (1, 1, 3, 6000, 2), (1, 1, 700, 513, 1), (1, 7, 50, 24, 8), (2, 2, 129, 65, 13),
]
OPTIONS = [(kavg.KAVG_ACT_NONE, 0.0), (kavg.KAVG_ACT_RELU, 0.25), (kavg.KAVG_ACT_SILU, 0.0), (kavg.KAVG_ACT_SILU, 0.1)]
EPS = 1e-5


def _inputs(shape, dtype, seed, offset=0.5):
    J, I, S, C, _ = shape
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, generator=gen, device="cuda")
    x = (normal(J, I, S, C) * (0.5 + torch.rand(J, 1, 1, C, generator=gen, device="cuda")) + offset * normal(J, 1, 1, C)).to(dtype)
    return x, normal(J, I, S, C).to(dtype), 1 + 0.3 * normal(J, C), 0.3 * normal(J, C)


def _np(t):
    return t.detach().cpu().double().numpy()


def _within(got, want, bound, dtype=torch.float32):
    got = _np(got)
    assert got.shape == want.shape
    if dtype is torch.bfloat16:
        bound = bound + 2.0 ** -8 * np.abs(want)
    off = np.abs(got - want) - bound
    assert not (off > 0).any() and np.isfinite(got).all(), "off by %.3g where %.3g is allowed" % (
        np.abs(got - want).flat[off.argmax()], np.broadcast_to(bound, off.shape).flat[off.argmax()])


def _steady(x, mean, rstd, w, b, groups, dy, act):
    """ReLU: no gradient where the pre-activation is so near zero that its sign is a matter of rounding."""
    if act != kavg.KAVG_ACT_RELU:
        return dy
    J, I, S, C = x.shape
    xg = _np(x).reshape(J, I, S, groups, -1)
    z = ((xg - _np(mean)[:, :, None, :, None]) * _np(rstd)[:, :, None, :, None]).reshape(x.shape) * _np(w)[:, None, None] + _np(b)[:, None, None]
    return torch.where(torch.from_numpy(np.abs(z) > 1e-4).cuda(), dy, torch.zeros_like(dy))


def _check(x, dy, w, b, groups, act, drop, seed=12345678901234567, site=3, make=lambda t: t, weight=None, bias=None, out=None):
    """make: the tensor that the call is given in place of a dense one."""
    f = R.keep_factors(tuple(x.shape), drop, seed, site)
    opt = dict(activation=act, drop=drop, seed=seed, site=site)
    weight, bias = (w if weight is None else weight), (b if bias is None else bias)
    y, mean, rstd = kavg.kavg_group_norm(make(x), weight, bias, groups, eps=EPS, stats=True, out=None if out is None else out(), **opt)
    want, m, r, bound = R.group_norm(_np(x), _np(w), _np(b), groups, EPS, act, f)
    _within(y, want, bound, x.dtype)
    spread = np.abs(_np(x)).max()
    assert np.abs(_np(mean) - m).max() <= R.K * spread
    assert (np.abs(_np(rstd) / r - 1) <= R.K * (1 + (spread * r) ** 2 * R.K)).all()
    assert torch.equal(kavg.kavg_group_norm(make(x), weight, bias, groups, eps=EPS, **opt), y)
    dy = _steady(x, mean, rstd, w, b, groups, dy, act)
    got = kavg.kavg_group_norm_backward(make(dy), make(x), mean, rstd, weight, bias, groups, out=None if out is None else out(), **opt)
    wants, bounds = R.group_norm_backward(_np(dy), _np(x), _np(mean), _np(rstd), _np(w), _np(b), groups, act, f)
    _within(got[0], wants[0], bounds[0], x.dtype)
    for k in (1, 2):
        _within(got[k], wants[k], bounds[k])
    again = kavg.kavg_group_norm_backward(make(dy), make(x), mean, rstd, weight, bias, groups, **opt)
    assert all(torch.equal(p, q) for p, q in zip(got, again))            # no order of sums left to chance
    return y, got


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s)))
def test_against_64_bits(shape, dtype):
    for k, (act, drop) in enumerate(OPTIONS):
        x, dy, w, b = _inputs(shape, dtype, 17 * k + shape[2])
        _check(x, dy, w, b, shape[4], act, drop)


# Many chunks for the lanes of few or many groups, packs of two halves in different groups, rows that are not whole lines, short and long,
# images that just fit a workgroup.
@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 1, 20000, 64, 64), (1, 1, 20000, 33, 33), (2, 3, 50, 40, 10), (1, 1, 20000, 40, 10), (1, 3, 784, 40, 5), (1, 1, 5000, 320, 32),
                                   (1, 1, 2048, 32, 4), (1, 1, 2049, 32, 4), (2, 300, 2, 16, 2), (1, 9, 1, 8, 8), (1, 2, 3, 8192, 1),
                                   (1, 3, 2, 16400, 1), (2, 2, 5, 9001, 1), (1, 2, 40, 1031, 1), (2, 3, 1, 12297, 3), (1, 1, 20000, 20, 5),
                                   (2, 3, 50, 36, 18), (1, 2, 300, 60, 12), (1, 1, 5000, 60, 12), (1, 3, 40, 380, 38), (3, 5, 16, 4, 2),
                                   (2, 3, 51, 22, 11), (1, 2, 300, 54, 2), (1, 1, 20001, 10, 5), (1, 1, 5000, 70, 14), (1, 40, 3, 2, 1)], ids=lambda s: "-".join(map(str, s)))
def test_edges_of_the_tiles(shape, dtype):
    for k, (act, drop) in enumerate(((kavg.KAVG_ACT_SILU, 0.1), (kavg.KAVG_ACT_RELU, 0.0))):
        x, dy, w, b = _inputs(shape, dtype, 31 * k + shape[2])
        _check(x, dy, w, b, shape[4], act, drop)


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(2, 3, 31, 24, 3), (1, 2, 1030, 64, 8), (2, 2, 20, 21, 3), (2, 2, 33, 20, 5), (2, 2, 33, 14, 7), (2, 2, 20, 1031, 1)], ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("pad,first", [(8, 0), (8, 8), (3, 1), (1, 0)])
def test_channels_of_a_wider_tensor(shape, dtype, pad, first):
    """x, dy and the output are channel slices of longer rows, whose other values stay what they are; images and sets lie apart."""
    J, I, S, C, G = shape
    x, dy, w, b = _inputs(shape, dtype, 5)

    def holder():
        return torch.full((J, 2 * I, S + 1, C + pad + first), 7.0, dtype=dtype, device="cuda")

    def place(whole):
        return whole[:, ::2, 1:, first:first + C]

    def make(t):
        whole = holder()
        place(whole).copy_(t)
        return place(whole)

    wholes = []

    def out():
        wholes.append(holder())
        return place(wholes[-1])

    _check(x, dy, w, b, G, kavg.KAVG_ACT_SILU, 0.2, make=make, out=out)
    for whole in wholes:
        place(whole).fill_(7.0)
        assert (whole == 7.0).all()


def test_parameters_inside_replicas():
    """Every learner's weight and bias lie in its flat replica, at an odd place; so do their gradients."""
    shape = (3, 4, 50, 24, 4)
    x, dy, w, b = _inputs(shape, torch.bfloat16, 6)
    flat, grad = torch.full((3, 101), 9.0, device="cuda"), torch.full((3, 103), 9.0, device="cuda")
    weight, bias = flat[:, 1:25], flat[:, 60:84]
    weight.copy_(w)
    bias.copy_(b)
    _, got = _check(x, dy, w, b, 4, kavg.KAVG_ACT_SILU, 0.0, weight=weight, bias=bias)
    _, mean, rstd = kavg.kavg_group_norm(x, weight, bias, 4, eps=EPS, activation=kavg.KAVG_ACT_SILU, stats=True)
    dw, db = grad[:, 3:27], grad[:, 30:54]
    kavg.kavg_group_norm_backward(dy, x, mean, rstd, weight, bias, 4, activation=kavg.KAVG_ACT_SILU, dweight=dw, dbias=db)
    assert torch.equal(dw, got[1]) and torch.equal(db, got[2])
    dw.fill_(9.0)
    db.fill_(9.0)
    assert (grad == 9.0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(2, 2, 9, 16, 4), (1, 1, 3000, 64, 8), (2, 1, 12, 1031, 1)], ids=str)
def test_without_parameters_and_one_set(shape, dtype):
    J, I, S, C, G = shape
    x, dy, _, _ = _inputs(shape, dtype, 7)
    one, zero = torch.ones(J, C, device="cuda"), torch.zeros(J, C, device="cuda")
    opt = dict(activation=kavg.KAVG_ACT_SILU, drop=0.1, seed=5)
    y, mean, rstd = kavg.kavg_group_norm(x, None, None, G, stats=True, **opt)
    assert torch.equal(y, kavg.kavg_group_norm(x, one, zero, G, **opt))
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, None, None, G, **opt)
    want = kavg.kavg_group_norm_backward(dy, x, mean, rstd, one, zero, G, **opt)
    assert dw is None and db is None and torch.equal(dx, want[0])
    only = kavg.kavg_group_norm_backward(dy, x, mean, rstd, one, None, G, **opt)
    assert torch.equal(only[1], want[1]) and only[2] is None
    # one learner without the dimension of sets
    flat = x.reshape(J * I, S, C)
    assert torch.equal(kavg.kavg_group_norm(flat, one[0], zero[0], G, **opt).view_as(y), y)


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 3, 40, 24, 3), (1, 2, 5000, 64, 8), (1, 1, 70, 21, 7), (1, 2, 90, 1031, 1)], ids=str)
def test_in_place(shape, dtype):
    x, dy, w, b = _inputs(shape, dtype, 8)
    opt = dict(activation=kavg.KAVG_ACT_SILU, drop=0.1, seed=5)
    y, mean, rstd = kavg.kavg_group_norm(x, w, b, shape[4], stats=True, **opt)
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, shape[4], **opt)
    g = dy.clone()
    at = kavg.kavg_group_norm_backward(g, x, mean, rstd, w, b, shape[4], out=g, **opt)
    assert torch.equal(g, dx) and torch.equal(at[1], dw) and torch.equal(at[2], db)
    z = x.clone()
    kavg.kavg_group_norm(z, w, b, shape[4], out=z, **opt)
    assert torch.equal(z, y)


def test_gradient_of_a_sum_is_a_broadcast_input():
    """dy with strides of 0 along sets, images and positions."""
    shape = (2, 3, 40, 16, 4)
    x, _, w, b = _inputs(shape, torch.float32, 9)
    row = torch.randn(16, device="cuda")
    _, mean, rstd = kavg.kavg_group_norm(x, w, b, 4, stats=True)
    got = kavg.kavg_group_norm_backward(row.expand(x.shape), x, mean, rstd, w, b, 4)
    want = kavg.kavg_group_norm_backward(row.expand(x.shape).contiguous(), x, mean, rstd, w, b, 4)
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", [(1, 3, 40, 20, 5), (1, 3, 1500, 64, 8), (1, 2, 35, 21, 7), (1, 3, 9000, 24, 4), (1, 3, 20, 2062, 2)], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_one_value_that_is_no_number_stays_in_its_group(shape, dtype, value):
    _, I, S, C, G = shape
    x, dy, w, b = _inputs(shape, dtype, 10)
    y0, m0, r0 = kavg.kavg_group_norm(x, w, b, G, stats=True)
    g0 = kavg.kavg_group_norm_backward(dy, x, m0, r0, w, b, G)
    D, hit = C // G, (C // (C // G)) // 2
    x[0, 1, S // 2, hit * D] = value
    y, mean, rstd = kavg.kavg_group_norm(x, w, b, G, stats=True)
    inside = torch.zeros_like(x, dtype=torch.bool)
    inside[0, 1, :, hit * D:(hit + 1) * D] = True
    assert torch.isnan(y[inside]).all() and torch.equal(y[~inside], y0[~inside])
    assert torch.isnan(rstd[0, 1, hit]) and torch.isfinite(rstd).sum() == I * G - 1
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, G)
    assert torch.isnan(dx[inside]).all() and torch.equal(dx[~inside], g0[0][~inside])
    channels = inside[0, 1, 0]
    assert torch.isnan(dw[0][channels]).all() and torch.equal(dw[0][~channels], g0[1][0][~channels])
    assert torch.equal(db[0][~channels], g0[2][0][~channels])


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
def test_constant_and_far_from_zero(dtype):
    """A group of equal values is its bias; values far from zero against their spread keep their variance."""
    w, b = torch.full((1, 64), 2.0, device="cuda"), torch.arange(64, device="cuda").float()[None]
    for S in (1, 50, 5000):
        x = torch.full((1, 2, S, 64), 3.5, dtype=dtype, device="cuda")
        y, mean, rstd = kavg.kavg_group_norm(x, w, b, 8, stats=True)
        assert torch.equal(y, b.to(dtype).expand(y.shape)) and (mean == 3.5).all()
    gen = torch.Generator(device="cuda").manual_seed(1)
    for S in (40, 5000):
        x = (1024 + 8 * torch.randint(-3, 4, (1, 2, S, 64), generator=gen, device="cuda")).to(dtype)     # (exact in bf16)
        y, _, _ = kavg.kavg_group_norm(x, w, b, 8, eps=EPS, stats=True)
        want, _, _, bound = R.group_norm(_np(x), _np(w), _np(b), 8, EPS, 0)
        _within(y, want, bound, dtype)


def test_nothing_to_normalise():
    w, b = torch.ones(2, 8, device="cuda"), torch.zeros(2, 8, device="cuda")
    for shape in ((2, 0, 5, 8), (2, 3, 0, 8)):
        x = torch.empty(shape, device="cuda")
        y, mean, rstd = kavg.kavg_group_norm(x, w, b, 2, stats=True)
        assert y.shape == x.shape and mean.shape == shape[:2] + (2,)
        dx, dw, db = kavg.kavg_group_norm_backward(x, x, mean, rstd, w, b, 2)
        assert dx.shape == x.shape and not dw.any() and not db.any()
    x = torch.empty(0, 3, 5, 8, device="cuda")
    e = torch.empty(0, 8, device="cuda")
    y, mean, rstd = kavg.kavg_group_norm(x, e, e, 2, stats=True)
    dx, dw, db = kavg.kavg_group_norm_backward(x, x, mean, rstd, e, e, 2)
    assert dw.shape == (0, 8) and dx.shape == x.shape


@pytest.mark.parametrize("act", [kavg.KAVG_ACT_NONE, kavg.KAVG_ACT_SILU])
def test_gradient_against_differences(act):
    """<dx, u> against (L(x + t u) - L(x - t u)) / 2t, L = <y, dy> in 64 bits of the library's own fp32 outputs.  A difference of two
    outputs is off by their roundings, 2^-22 |y dy| / t in the worst case summed like a random walk (a factor of 8 to be clear), and by
    t^2/6 of a third derivative, of the size of the gradient itself here."""
    shape = (1, 2, 30, 24, 4)
    x, dy, w, b = _inputs(shape, torch.float32, 11, offset=0.2)
    opt = dict(activation=act, drop=0.2, seed=77)
    _, mean, rstd = kavg.kavg_group_norm(x, w, b, 4, stats=True, **opt)
    dx, dw, db = kavg.kavg_group_norm_backward(dy, x, mean, rstd, w, b, 4, **opt)
    gen = torch.Generator(device="cuda").manual_seed(12)
    t = 2.0 ** -7

    def loss(x, w, b):
        return float((kavg.kavg_group_norm(x, w, b, 4, **opt).double() * dy.double()).sum())

    for g, at in ((dx, 0), (dw, 1), (db, 2)):
        u = torch.randn(g.shape, generator=gen, device="cuda")
        sides = []
        for s in (1, -1):
            args = [x, w, b]
            args[at] = args[at] + s * t * u
            sides.append(loss(*args))
        y = kavg.kavg_group_norm(x, w, b, 4, **opt)
        allowed = 8 * 2.0 ** -22 * float((y * dy).double().norm()) / t + t * t * float((g.double() * u.double()).norm()) * 8
        assert abs((sides[0] - sides[1]) / (2 * t) - float((g.double() * u.double()).sum())) <= allowed


def test_on_a_side_stream_and_under_a_graph():
    """Work goes to the current stream; a recorded call replays with what its tensors hold then, beside the program's own work."""
    shape = (2, 2, 3000, 32, 4)
    x, dy, w, b = _inputs(shape, torch.bfloat16, 13)
    opt = dict(activation=kavg.KAVG_ACT_SILU, drop=0.1, seed=3)
    gx, gdy = torch.zeros_like(x), torch.zeros_like(dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        slow = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            slow = slow @ slow * 1e-2
        gx.copy_(x)
        gdy.copy_(dy)
        y, mean, rstd = kavg.kavg_group_norm(gx, w, b, 4, stats=True, **opt)
        grads = kavg.kavg_group_norm_backward(gdy, gx, mean, rstd, w, b, 4, **opt)
    side.synchronize()
    want = kavg.kavg_group_norm(x, w, b, 4, **opt)
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, mean, rstd = kavg.kavg_group_norm(gx, w, b, 4, stats=True, **opt)
        grads = kavg.kavg_group_norm_backward(gdy, gx, mean, rstd, w, b, 4, **opt)
    for k in range(4):
        x, dy, _, _ = _inputs(shape, torch.bfloat16, 14 + k)
        gx.copy_(x)
        gdy.copy_(dy)
        graph.replay()
        torch.cuda.synchronize()
        ey, em, er = kavg.kavg_group_norm(x, w, b, 4, stats=True, **opt)
        eager = kavg.kavg_group_norm_backward(dy, x, em, er, w, b, 4, **opt)
        assert torch.equal(y, ey) and torch.equal(mean, em) and torch.equal(rstd, er)
        assert all(torch.equal(p, q) for p, q in zip(grads, eager))
