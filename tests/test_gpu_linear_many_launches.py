"""Products of more tiles than a launch takes: 2^22 of 64 x 64 here, so more learners than that of a layer of single elements, or 2^28 rows."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L
from tests.test_gpu_linear import CODE, DTYPES, IDS, in_rows, normal

pytestmark = pytest.mark.gpu

LAUNCH = 1 << 22


def check(got, want, parts):
    """got and what `want(slice)` gives with its bound, part by part."""
    for part in parts:
        for g, e in zip([None if t is None else t[part] for t in got], want(part)):
            L.close(g, e)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
def test_millions_of_learners(turned, dtype):
    """Everything of a learner moves on by learners: weights, biases, residuals, pre-activations, all three gradients.  A learner's results are those of a call of few
    learners to the last bit; around the borders they are compared with 64 bits."""
    J, M, K, N = LAUNCH + 5, 1, 3, 1
    x, w, b, r = normal(1, J, M, K, dtype=dtype), in_rows(normal(2, J, N, K, dtype=dtype), turned, 1), normal(3, J, N), normal(4, J, M, N, dtype=dtype)
    pre = normal(5, J, M, K, dtype=dtype)
    forward = lambda x, w, b, r: kavg.kavg_linear(x, w, b, activation=CODE["silu"], residual=r, pre=True)  # noqa: E731
    for other in (None, torch.empty(J, K, N, device="cuda").transpose(1, 2)):
        got = [*forward(x, w, b, r), *kavg.kavg_linear_backward(r, x, w, activation=CODE["silu"], pre=pre, dweight=other)]

        def want(part):
            return [*L.linear(x[part], w[part], b[part], "silu", r[part], dtype), *L.linear_backward(r[part], x[part], w[part], "silu", pre[part], dtype)]
        check(got, want, (slice(0, 40), slice(LAUNCH - 40, None)))
        half = J // 2
        for part in (slice(0, half), slice(half, None)):
            again = [*forward(x[part], w[part], b[part], r[part]), *kavg.kavg_linear_backward(r[part], x[part], w[part], activation=CODE["silu"], pre=pre[part],
                                                                                              dweight=None if other is None else torch.empty(len(x[part]), K, N, device="cuda").transpose(1, 2))]
            assert all(torch.equal(a[part], e) for a, e in zip(got, again))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_hundreds_of_millions_of_rows(dtype):
    """Everything of a row moves on by rows, in tensors of more than 2^31 bytes; the weight's and the bias's gradients are one contraction."""
    border = LAUNCH * 64
    M, K, N = border + 70, 3, 1
    x, w, b, r = normal(1, M, K, dtype=dtype), normal(2, N, K, dtype=dtype), normal(3, N), normal(4, M, N, dtype=dtype)
    y, z = kavg.kavg_linear(x, w, b, activation=CODE["relu"], residual=r, pre=True)
    dx = kavg.kavg_linear_backward(r, x, w, activation=CODE["relu"], pre=x, dweight=False, dbias=False)[0]
    parts = [slice(0, 1 << 20), slice(border - (1 << 20), None)]
    check((y, z), lambda part: L.linear(x[part], w, b, "relu", r[part], dtype), parts)
    check((dx,), lambda part: L.linear_backward(r[part], x[part], w, "relu", x[part], dtype)[:1], parts)
    half = M // 2
    for part in (slice(0, half), slice(half, None)):
        assert torch.equal(y[part], kavg.kavg_linear(x[part], w, b, activation=CODE["relu"], residual=r[part]))
