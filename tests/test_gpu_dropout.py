"""kavg_dropout and its backward pass: the mask bit for bit, the values within a rounding."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import layers_reference as R

pytestmark = pytest.mark.gpu

DTYPES = (torch.float32, torch.bfloat16)
SHAPES = [(1, 1), (1, 3), (7, 1), (1, 4097), (3, 5), (5, 8), (33, 12), (64, 256), (100, 1001), (17, 2040), (2, 70001), (1000, 3), (513, 64)]


def _x(shape, dtype, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _want(x, f, residual, dtype):
    """A product with the scale (itself rounded to fp32) and a sum in fp32: three roundings; one more in bf16."""
    v = x.double().cpu().numpy() * f
    size = np.abs(v)
    if residual is not None:
        r = residual.double().cpu().numpy()
        v, size = v + r, size + np.abs(r)
    bound = 3 * 2.0 ** -24 * size
    return v, bound + (2.0 ** -8 * np.abs(v) if dtype is torch.bfloat16 else 0)


def _close(y, want, bound):
    assert (np.abs(y.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("drop", [0.0, 0.1, 0.5, 0.99, 1.0])
def test_values_and_mask(shape, dtype, drop):
    x, residual = _x(shape, dtype), _x(shape, dtype, 2)
    seed, site = 0xFEDCBA9876543210, (1 << 24) - 1
    f = R.keep_factors(shape, drop, seed, site)
    y = kavg.kavg_dropout(x, drop, seed, site=site)
    _close(y, *_want(x, f, None, dtype))
    assert np.array_equal(y.double().cpu().numpy() != 0, (f != 0) & (x != 0).cpu().numpy())
    assert torch.equal(kavg.kavg_dropout_backward(x, drop, seed, site=site), y)
    _close(kavg.kavg_dropout(x, drop, seed, site=site, residual=residual), *_want(x, f, residual, dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("rows,cols,pad,first", [(9, 64, 8, 0), (9, 64, 8, 8), (9, 64, 3, 1), (30, 21, 4, 2), (31, 12, 1, 0), (4, 1000, 24, 0), (300, 2, 1, 0)])
def test_rows_apart(rows, cols, pad, first, dtype):
    """x, residual and the output are slices of longer rows, at any alignment; what lies between stays."""
    f = R.keep_factors((rows, cols), 0.3, 5, 1)

    def place(whole):
        return whole[:, first:first + cols]

    x, residual = place(_x((rows, cols + pad + first), dtype)), place(_x((rows, cols + pad + first), dtype, 2))
    whole = torch.full((rows, cols + pad + first), 7.0, dtype=dtype, device="cuda")
    y = kavg.kavg_dropout(x, 0.3, 5, site=1, residual=residual, out=place(whole))
    _close(y, *_want(x, f, residual, dtype))
    place(whole).fill_(7.0)
    assert (whole == 7.0).all()
    _close(kavg.kavg_dropout_backward(x, 0.3, 5, site=1), *_want(x, f, None, dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
@pytest.mark.parametrize("first", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 1023, 40000])
def test_any_start_and_length(n, first, dtype):
    whole = _x(n + 16, dtype)
    x = whole[first:first + n]
    f = R.keep_factors((n,), 0.4, 8, 2)
    target = torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")
    y = kavg.kavg_dropout(x, 0.4, 8, site=2, out=target[3:3 + n])
    _close(y, *_want(x, f, None, dtype))
    assert (target[:3] == 7.0).all() and (target[3 + n:] == 7.0).all()


def test_shapes_of_any_rank_and_broadcast_inputs():
    x = _x((3, 4, 5, 8), torch.float32)
    want = kavg.kavg_dropout(x.view(60, 8), 0.5, 1)
    assert torch.equal(kavg.kavg_dropout(x, 0.5, 1).view(60, 8), want)
    one = torch.ones((), device="cuda")
    assert kavg.kavg_dropout(one, 0.0, 1).item() == 1
    row = _x((8,), torch.float32)
    assert torch.equal(kavg.kavg_dropout_backward(row.expand(60, 8), 0.5, 1), kavg.kavg_dropout_backward(row.expand(60, 8).contiguous(), 0.5, 1))
    for shape in ((0, 8), (8, 0), (0,)):
        assert kavg.kavg_dropout(torch.empty(shape, device="cuda"), 0.5, 1).shape == shape


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
def test_infinities_and_nan_in_dropped_places(dtype):
    f = R.keep_factors((50, 37), 0.5, 4, 0)
    gone = torch.from_numpy(f == 0).cuda()
    for v in (float("inf"), float("nan"), -float("inf")):
        x = torch.where(gone, torch.full((50, 37), v, device="cuda"), torch.ones(50, 37, device="cuda")).to(dtype)
        y = kavg.kavg_dropout(x, 0.5, 4)
        assert (y[gone] == 0).all() and (y[~gone] == 2).all()
        assert (kavg.kavg_dropout(x, 1.0, 4) == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=("f32", "bf16"))
def test_in_place(dtype):
    for shape in ((64, 128), (7, 33)):
        x, residual = _x(shape, dtype), _x(shape, dtype, 2)
        want = kavg.kavg_dropout(x, 0.2, 9, residual=residual)
        a, r = x.clone(), residual.clone()
        kavg.kavg_dropout(a, 0.2, 9, residual=residual, out=a)
        kavg.kavg_dropout(x, 0.2, 9, residual=r, out=r)
        assert torch.equal(a, want) and torch.equal(r, want)


def test_elements_past_32_bits():
    """More than 2^32 elements: the last ones go by their own numbers, not by those modulo 2^32."""
    n = (1 << 32) + 40
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    kavg.kavg_dropout(x, 0.5, 6, out=x)
    e = np.arange(n - 64, n, dtype=np.uint64)
    with np.errstate(over="ignore"):
        z = R.mix(np.uint64(6) + (np.uint64(1) + e // np.uint64(4)) * np.uint64(0x9E3779B97F4A7C15))
    kept = ((z >> (np.uint64(16) * (e % np.uint64(4)))) & np.uint64(0xFFFF)) >= 32768
    assert np.array_equal(x[-64:].float().cpu().numpy(), np.where(kept, 2.0, 0.0))


def test_rate_and_independence():
    y = kavg.kavg_dropout(torch.ones(1 << 22, device="cuda"), 0.25, 123)
    kept = (y != 0).double()
    sd = (0.25 * 0.75 / kept.numel()) ** 0.5
    assert abs(float(kept.mean()) - 0.75) < 5 * sd and abs(float(y.double().mean()) - 1) < 5 * sd / 0.75
    for lag in (1, 2, 4, 64):
        c = (kept[lag:] - 0.75) * (kept[:-lag] - 0.75)
        assert abs(float(c.mean())) < 5 * 0.1875 / c.numel() ** 0.5
    other = (kavg.kavg_dropout(torch.ones(1 << 22, device="cuda"), 0.25, 124) != 0).double()
    assert abs(float(((other - 0.75) * (kept - 0.75)).mean())) < 5 * 0.1875 / kept.numel() ** 0.5


def test_on_a_side_stream_and_under_a_graph():
    x, residual = _x((300, 77), torch.bfloat16), _x((300, 77), torch.bfloat16, 2)
    gx, gr = torch.zeros_like(x), torch.zeros_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        slow = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            slow = slow @ slow * 1e-2
        gx.copy_(x)
        gr.copy_(residual)
        y = kavg.kavg_dropout(gx, 0.3, 2, residual=gr)
    side.synchronize()
    assert torch.equal(y, kavg.kavg_dropout(x, 0.3, 2, residual=residual))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = kavg.kavg_dropout(gx, 0.3, 2, residual=gr)
    for k in range(4):
        x, residual = _x((300, 77), torch.bfloat16, 10 + k), _x((300, 77), torch.bfloat16, 20 + k)
        gx.copy_(x)
        gr.copy_(residual)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, kavg.kavg_dropout(x, 0.3, 2, residual=residual))
