"""The layers' plain forms: the counter stream against the published vector, the gradients against differences."""
import os

import numpy as np
import pytest

from tests import layers_reference as R


def test_counter_stream_is_splitmix64():
    """Elements 4q .. 4q+3 hold the quarters of output number q + 1 (site 0), low bits first."""
    path = os.path.join(os.path.dirname(__file__), "golden", "splitmix64_seed1234567.txt")
    words = [int(line) for line in open(path).read().split() if line.strip().isdigit()][:5]
    assert len(words) == 5
    for t in (1, 100, 30000, 65535):
        kept = R.keep_factors((20,), t / 65536, 1234567, 0) != 0
        want = [(w >> (16 * i) & 0xFFFF) >= t for w in words for i in range(4)]
        assert np.array_equal(kept, want)
    assert not R.keep_factors((20,), 1.0, 3, 0).any()
    assert (R.keep_factors((20,), 0.0, 3, 0) == 1).all()
    sites = [R.keep_factors((4096,), 0.5, 9, s) for s in range(3)]
    assert all(0.4 < np.mean(a != b) < 0.6 for a, b in zip(sites, sites[1:]))
    assert abs(R.keep_factors((1 << 18,), 0.3, 5, 1).mean() - 1) < 5e-3          # 1/(1-p) keeps the expectation


@pytest.mark.parametrize("kind", (R.ACT_NONE, R.ACT_RELU, R.ACT_SILU))
@pytest.mark.parametrize("drop", (0.0, 0.3))
def test_gradients_against_differences(kind, drop):
    rng = np.random.default_rng(3)
    J, I, S, C, G, eps = 2, 3, 5, 12, 3, 1e-3
    x, dy = rng.normal(size=(2, J, I, S, C)) + 0.3
    w, b = rng.normal(size=(2, J, C)) + 0.5
    f = R.keep_factors(x.shape, drop, 11, 2)

    def loss(x, w, b):
        return float((R.group_norm(x, w, b, G, eps, kind, f)[0] * dy).sum())

    _, mean, rstd, _ = R.group_norm(x, w, b, G, eps, kind, f)
    (dx, dw, db), _ = R.group_norm_backward(dy, x, mean, rstd, w, b, G, kind, f)
    t = 1e-6
    for _ in range(4):
        u, uw, ub = rng.normal(size=x.shape), rng.normal(size=w.shape), rng.normal(size=b.shape)
        for got, step in (((dx * u).sum(), (u, 0, 0)), ((dw * uw).sum(), (0, uw, 0)), ((db * ub).sum(), (0, 0, ub))):
            ahead, back = (loss(x + s * t * step[0], w + s * t * step[1], b + s * t * step[2]) for s in (1, -1))
            assert abs((ahead - back) / (2 * t) - got) < 1e-5 * (1 + abs(got))
