"""Minibatch indices and dropout masks are drawn by one generator.  With one seed, learner j's first indices and the first words of site
j's mask are the same; with different seeds, as the interface asks for, they are not."""
import numpy as np

from oracle.mavg_oracle import minibatch_indices
from tests import layers_reference as R


def _fields(seed, site, words):
    """The lowest 16 bits of the words that a mask is drawn from."""
    c = np.arange(words, dtype=np.uint64) + np.uint64(1) + np.uint64(site) * np.uint64(1 << 40)
    with np.errstate(over="ignore"):
        return (R.mix(np.uint64(seed) + c * np.uint64(0x9E3779B97F4A7C15)) & np.uint64(0xFFFF)).astype(np.int64)


def test_one_seed_is_one_stream():
    for j in (0, 3):
        assert np.array_equal(minibatch_indices(11, j, 0, 64, 1 << 16), _fields(11, j, 64))


def test_two_seeds_are_two():
    for seed, other in ((11, 12), (0, 1), (5, 5 + (1 << 32))):
        assert (minibatch_indices(seed, 3, 0, 64, 1 << 16) == _fields(other, 3, 64)).sum() <= 2
