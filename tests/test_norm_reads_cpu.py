"""What the lanes of a group norm read (csrc/norm_tile.h, tile_load), on the host: no element outside a tensor whose images, sets or
positions share memory, in either direction, for the tiles that the library itself takes for such a call."""
import ctypes
import itertools

import numpy as np
import pytest

from tests import test_norm_tiles_cpu as tiles
from tests.test_norm_tiles_cpu import tiles_of  # noqa: F401  (loads the library)


def _call_tiles(lib, bf16, shape, x, dy, backward):
    """The library's choice for dense results; x, dy: strides of sets, images and positions."""
    sets, images, positions, channels, groups = shape
    dense = tiles.Strides(images * positions * channels, positions * channels, channels)
    c = tiles.NormCall(dtype=int(bf16), sets=sets, images=images, positions=positions, channels=channels, groups=groups, xs=tiles.Strides(*x),
                       dys=tiles.Strides(*dy), outs=dense)
    t = tiles.NormTiles()
    rule = lib._ZN4kavg10call_tilesERKNS_8NormCallEbPNS_9NormTilesE
    rule.restype = ctypes.c_bool
    rule.argtypes = [ctypes.POINTER(tiles.NormCall), ctypes.c_bool, ctypes.POINTER(tiles.NormTiles)]
    return t if rule(ctypes.byref(c), backward, ctypes.byref(t)) else None


def _extent(shape, strides):
    return sum((n - 1) * s for n, s in zip(shape, strides)) + shape[3]


def _lowest_and_highest(t, shape, strides):
    """The first and the last element that any lane asks for."""
    sets, images, positions, channels, _ = shape
    V, extent, low, high = t.vec, _extent(shape, strides), 0, -1
    first = {}
    for k, (image, start, n, _, channel) in enumerate(tiles._walk(t, shape, 1024)):
        base = image // images * strides[0] + image % images * strides[1]
        own = start if t.flat else start // channels * strides[2] + start % channels
        pack = k % t.nv
        if pack == 0:
            first = np.where(n > 0, base + own, base + (0 if t.flat else np.where(channel < channels, channel, 0)))
        at = np.where(n > 0, base + own, first)                  # (a lane without a pack asks for its first one again)
        if t.flat:
            high = max(high, int(np.minimum(at + V, extent).max()) - 1)
            at = np.where(at + V <= extent, at, extent - V)
        low, high = min(low, int(at.min())), max(high, int(at.max()) + V - 1)
    return low, high, extent


SHAPES = [(1, 9, 1, 1, 1), (1, 64, 1, 5, 1), (1, 3, 1, 3, 1), (3, 3, 1, 3, 3), (2, 5, 1, 7, 7), (1, 300, 1, 5, 5), (4, 2, 2, 3, 1), (2, 9, 7, 1, 1), (1, 2, 3, 9, 3),
          (2, 2, 33, 5, 1), (1, 3, 20000, 3, 1), (1, 6, 1, 6, 2), (2, 9, 1, 8, 2), (3, 4, 5, 12, 3)]


@pytest.mark.parametrize("bf16,backward", list(itertools.product((False, True), repeat=2)))
def test_no_element_outside_a_tensor(tiles_of, bf16, backward):  # noqa: F811
    from paper_2110_00625_amd import kavg
    lib, flat = kavg.load_library(), 0
    for shape in SHAPES:
        sets, images, positions, channels, _ = shape
        dense = (images * positions * channels, positions * channels, channels)
        some = [dense, (0, 0, channels), (0, 1, channels), (1, 0, channels), (dense[0], 0, channels), (0, dense[1], channels), (2, 1, channels), (0, 0, 0), (1, 1, 1),
                (dense[0] + 5, dense[1] + 1, channels), (dense[1], sets * dense[1], channels)]
        if positions == 1:                                   # (the stride says nothing; the library sets it)
            some = [(a, b, channels) for a, b, _ in some]
        for x, dy in itertools.product(some, some if backward else [dense]):
            t = _call_tiles(lib, bf16, shape, x, dy, backward)
            if t is None:
                continue
            for u in (t.whole,) if t.whole.nv else (t.sums, t.apply):
                flat += u.flat
                for strides in (x, dy) if backward else (x,):
                    low, high, extent = _lowest_and_highest(u, shape, strides)
                    assert low >= 0 and high < extent, "%s, strides %s: elements %d .. %d of %d" % (shape, strides, low, high, extent)
    assert flat > 20
