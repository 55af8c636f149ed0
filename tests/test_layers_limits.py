"""The limits of the layers that include/kavg.h names, from both sides, at the C boundary before any device call."""
import ctypes

import pytest

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import AT, backward, forward, images, lib, norm  # noqa: F401  (lib: the loaded library)


def _accepted(lib, **kw):  # noqa: F811
    size, codes = ctypes.c_size_t(0), []
    for direction in (0, 1):
        codes.append(lib.kavg_group_norm_workspace(norm(**kw), direction, ctypes.byref(size)))
    assert codes[0] == codes[1]
    return codes[0] == kavg.KAVG_OK


@pytest.mark.parametrize("over,within", [
    (dict(sets=1, images=1 << 27, positions=1, channels=64, groups=16), dict(sets=1, images=(1 << 27) - 1, positions=1, channels=64, groups=16)),
    (dict(sets=1 << 20, images=1 << 11, positions=1, channels=2, groups=1), dict(sets=1 << 20, images=(1 << 11) - 1, positions=1, channels=2, groups=1)),
    (dict(sets=1 << 20, images=1, positions=1, channels=1 << 11, groups=1), dict(sets=1 << 20, images=1, positions=1, channels=(1 << 11) - 1, groups=1)),
    (dict(sets=1, images=1, positions=1 << 32, channels=1 << 10, groups=2), dict(sets=1, images=1, positions=(1 << 32) - 1, channels=1 << 10, groups=2)),
    (dict(sets=0, images=1 << 28, positions=1, channels=8, groups=8), dict(sets=0, images=1 << 27, positions=1, channels=8, groups=8)),
])
def test_sizes(lib, over, within):  # noqa: F811
    assert not _accepted(lib, **over) and _accepted(lib, **within)
    n = norm(**over)
    assert forward(lib, n) == kavg.KAVG_EINVAL and backward(lib, n) == kavg.KAVG_EINVAL


def test_strides(lib):  # noqa: F811
    """Two learners of three images of four positions: a stride past its limit is refused, one at it is not (the call then ends at its
    workspace, which is not there)."""
    E, most = kavg.KAVG_EINVAL, [(1 << 46) // n for n in (2, 3, 4)]

    def call(x, w=8):
        n = norm(positions=4, channels=8, groups=2)
        return lib.kavg_group_norm_backward(n, x, x, AT, AT, AT, w, AT, 8, images(), AT, 8, AT, 8, None, 0, None)
    assert call(images()) == kavg.KAVG_ENOMEM
    for k in range(3):
        for past, code in ((0, kavg.KAVG_ENOMEM), (1, E)):
            strides = [96, 32, 8]
            strides[k] = most[k] + past
            assert call(kavg._IMAGES.pack(AT, *strides)) == code
    assert call(images(), w=(1 << 46) // 2) == kavg.KAVG_ENOMEM and call(images(), w=(1 << 46) // 2 + 1) == E


def test_strides_of_dropout(lib):  # noqa: F811
    def drop(xs=8, rs=8, ys=8, rows=4, cols=8):
        return lib.kavg_dropout(AT, xs, AT, rs, AT, ys, rows, cols, 0, 0.5, 1, 0, None)
    for kw in (dict(xs=(1 << 44) + 1), dict(rs=(1 << 44) + 1), dict(ys=(1 << 44) + 1), dict(cols=1 << 30, xs=0, rs=0, ys=1 << 30)):
        assert drop(**kw) == kavg.KAVG_EINVAL, kw


def test_channels(lib):  # noqa: F811
    """Channels are counted in 32 bits by workgroups that go a little past the last one."""
    for sets, groups in ((1, 1), (1, 1 << 10), (0, 1)):
        most = (1 << 31) - (1 << 16)
        assert _accepted(lib, sets=sets, images=1, positions=1, channels=most, groups=groups)
        for over in (most + (1 << 10), (1 << 31) - (1 << 10)):
            kw = dict(sets=sets, images=1, positions=1, channels=over, groups=groups)
            assert not _accepted(lib, **kw)
            assert forward(lib, norm(**kw)) == kavg.KAVG_EINVAL and backward(lib, norm(**kw)) == kavg.KAVG_EINVAL
