"""The bias's gradient over many rows.

A run of the kernel's fp32 sums is 2048 rows and as many more as the last slices are, at most 4 of 64: each of its sums has at most (2048 + 256) / 8 additions of a term
or of two (an operand's two halves in four sums each), good for two units of 2^-24 of the magnitudes each should an addition cut instead of round; three more join the
eight sums.  Runs are added in 64 bits.  A part is rounded once to fp32, at most 32 parts are added in fp32.  In all 2 (288 + 3) + 1 + 32 units of 2^-24 of
the sum of the magnitudes, however many rows there are."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L
from tests.test_gpu_linear import DTYPES, IDS, normal

pytestmark = pytest.mark.gpu

UNITS = 2 * (288 + 3) + 1 + 32


def close(db, dz):
    want = torch.zeros(db.shape, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    for part in dz.split(1 << 22, -2):
        want += part.double().sum(-2)
        size += part.double().abs().sum(-2)
    off = (db.double() - want).abs() / (UNITS * L.U * size)
    assert float(off.max()) <= 1, "off by %.3g of the bound" % float(off.max())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("values", ("one", "spread"))
@pytest.mark.parametrize("sets,rows,outputs", [(1, 1 << 23, 8), (1, (1 << 23) + 77, 5), (3, 1 << 21, 40), (2, 3_000_001, 1), (1, (1 << 27) + 5, 1)], ids=str)
def test_millions_of_rows(sets, rows, outputs, values, dtype):
    """One value throughout, whose roundings add up while a sum stays in a binade, and values of one sign."""
    if values == "one":
        dz = torch.linspace(0.1, 0.9, outputs, device="cuda").to(dtype).expand(sets, rows, outputs).contiguous()
    else:
        dz = normal(1, sets, rows, outputs).abs().to(dtype)
    w = torch.zeros(sets, outputs, 8, dtype=dtype, device="cuda")
    x = torch.zeros(sets, rows, 8, dtype=dtype, device="cuda")
    alone = kavg.kavg_linear_backward(dz, x, w, out=False, dweight=False)[2]
    close(alone, dz)
    for dweight in (None, torch.empty(sets, 8, outputs, device="cuda").transpose(1, 2)):
        close(kavg.kavg_linear_backward(dz, x, w, out=False, dweight=dweight)[2], dz)


# sets, rows, inputs, outputs: 256 x 256, 128 x 128, 128 x 128 through registers, 64 x 64 not split
@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size", [(1, 1 << 16, 4096, 4096), (1, 1 << 16, 2048, 2048), (1, 1 << 16, 2047, 2047), (8, 1 << 16, 512, 512)], ids=str)
@pytest.mark.parametrize("other", (False, True), ids=("", "turned"))
def test_every_tile(size, other, dtype):
    J, M, K, N = size
    dz = torch.linspace(0.1, 0.9, N, device="cuda").to(dtype).expand(J, M, N).contiguous()
    dz[:, ::2] = dz[:, ::2] * 0.75
    x, w = normal(2, J, M, K, dtype=dtype), torch.zeros(J, N, K, dtype=dtype, device="cuda")
    dweight = torch.empty(J, K, N, device="cuda").transpose(1, 2) if other else None
    _, dw, db = kavg.kavg_linear_backward(dz, x, w, out=False, dweight=dweight)
    close(db, dz)
    # (columns of the product beside it: a sum of M products in fp32)
    some = torch.arange(0, N, 97, device="cuda")
    L.close(dw[:, some], L.product(dz[:, :, some].transpose(1, 2), x.transpose(1, 2)))
