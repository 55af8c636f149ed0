"""Products of every kind of tile against 64 bits, at contractions of many slices: with and without the loop of whole slices, a last slice in part, split and
not, straight into LDS and through registers.  What a size is there for, by the products' cost rule (dx and dW of plain weights):"""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L
from tests.test_gpu_linear import CODE, DTYPES, IDS, in_rows, normal, operands

pytestmark = pytest.mark.gpu

# sets, rows, inputs, outputs
SIZES = [
    # 256 x 256, bf16: forward; dx; dW of 16 slices, of two, of three whose last is in part; split: dW, dx, forward, the last slices in part
    (1, 4096, 512, 4096), (1, 4096, 4096, 520), (1, 1024, 4096, 4096), (16, 128, 1024, 1024), (1, 136, 30744, 432), (3, 6544, 6064, 200), (1, 240, 21088, 5160), (2, 200, 4792, 10704),
    # the same in fp32, split: dW, dx, forward
    (1, 5168, 1264, 17376), (2, 2560, 4352, 6144), (1, 2552, 5072, 8680),
    # 128 x 128: all three, aligned and not; split: dW, dx, forward in bf16, through registers, in fp32, through registers
    (4, 1000, 1000, 1000), (4, 1001, 1001, 1001), (3, 7984, 72, 1064), (1, 1384, 80, 16912), (3, 2784, 3704, 72), (1, 5585, 72, 4243), (1, 9579, 67, 3022), (1, 67, 8394, 4924),
    (1, 656, 72, 8872), (2, 2296, 72, 1544), (1, 8560, 768, 80), (1, 727, 65, 9544), (1, 2776, 72, 2055), (3, 2736, 665, 67),
    # 64 x 64, with a ring of four slices, split and not
    (1, 64, 696, 64), (1, 64, 10944, 64), (1, 1867, 64, 84), (1, 118, 1686, 65),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
def test_long_contractions(size, dtype, turned):
    x, w, b, dz = operands(size, dtype)
    at = in_rows(w, turned)
    y, z = kavg.kavg_linear(x, at, b, activation=CODE["silu"], residual=dz, pre=True)
    want_y, want_z = L.linear(x, w, b, "silu", dz, dtype)
    L.close(y, want_y)
    L.close(z, want_z)
    del y, z, want_y, want_z
    pre = normal(9, *x.shape, dtype=dtype)
    for got, want in zip(kavg.kavg_linear_backward(dz, x, at, activation=CODE["relu"], pre=pre), L.linear_backward(dz, x, w, "relu", pre, dtype)):
        L.close(got, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,n", [(40, 64), (200, 512), (8192, 256), (2048, 1024), (4096, 2048), (16384, 1024), (515, 1003)], ids=str)
def test_results_stay_in_their_places(rows, n, dtype):
    """Products with a permutation: every result is one value of the other operand, whole numbers that neighbours within 200 rows and columns do not share, to the
    last bit.  A result that left from another lane's place, or from the block before, would be another number."""
    x = ((torch.arange(rows, device="cuda")[:, None] * 17 + torch.arange(n, device="cuda") * 29) % 251).to(dtype)
    order = torch.randperm(n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    w = torch.eye(n, device="cuda")[order].to(dtype)
    for at in (w, w.t().contiguous().t()):
        y, z = kavg.kavg_linear(x, at, activation=CODE["relu"], pre=True)
        assert torch.equal(y, x[:, order]) and torch.equal(z, y)
        assert torch.equal(kavg.kavg_linear_backward(y, x, at, dweight=False, dbias=False)[0], x)
    pick = torch.randperm(rows, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")[:min(rows, n)]
    one = torch.zeros(rows, pick.numel(), dtype=dtype, device="cuda")
    one[pick, torch.arange(pick.numel(), device="cuda")] = 1
    for dw in (None, torch.empty(n, pick.numel(), device="cuda").t()):
        got = kavg.kavg_linear_backward(one, x, torch.zeros(pick.numel(), n, dtype=dtype, device="cuda"), out=False, dweight=dw)
        assert torch.equal(got[1], x[pick].float()) and (got[2] == 1).all()
