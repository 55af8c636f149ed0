"""Packs per lane of a group norm's tiles (csrc/norm_tile.hip), on the host: where a lane has several, more than half of a workgroup's
are the image's, however many images there are.  (A lane without a pack asks for another's and works out results that go nowhere.)"""
import itertools

import pytest

from tests.test_norm_tiles_cpu import tiles_of  # noqa: F401  (loads the library)

CHANNELS = [(1024, 16), (4096, 16), (512, 16), (96, 8), (64, 8), (12, 3), (91, 7), (33, 3), (5, 1), (1, 1)]


@pytest.mark.parametrize("bf16,backward,contiguous", list(itertools.product((False, True), repeat=3)))
def test_lanes_have_no_packs_that_do_not_exist(tiles_of, bf16, backward, contiguous):  # noqa: F811
    several = 0
    for (channels, groups), positions, images in itertools.product(CHANNELS, (1, 2, 3, 6, 9, 16, 49, 196, 1000),
                                                                   (1, 100, 1000, 1024, 2047, 2048, 4096, 60000, 1 << 20)):
        t = tiles_of(bf16, (1, images, positions, channels, groups), contiguous, backward)
        if t is None or t.whole.nv <= 1:
            continue
        several += 1
        t = t.whole
        packs = -(-positions * channels // t.vec) if t.flat else positions * t.cols
        assert 2 * packs > t.nv * t.cols * t.lane_rows, "%d images of %d positions, %d channels: %d packs for %d lanes of %d" % (
            images, positions, channels, packs, t.cols * t.lane_rows, t.nv)
    assert several > 50
