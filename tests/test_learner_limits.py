"""Limits of the learners' calls at the C boundary, before any device call (no GPU needed)."""
import numpy as np

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import lib  # noqa: F401  (lib: the loaded library)
from tests.test_learner_refusals import adamw

E, OK = kavg.KAVG_EINVAL, kavg.KAVG_OK


def test_numbers_past_fp32(lib):  # noqa: F811
    """A rate or a factor that is infinite in fp32 would make NaN of a gradient or a moment of 0."""
    most = float(np.finfo(np.float32).max)
    for ok in (dict(lr=most), dict(grad_scale=most), dict(grad_scale=-most), dict(eps=1e300), dict(eps=1e-300)):
        assert adamw(lib, ok) == OK, ok
    for wrong in (dict(lr=1.0001 * most), dict(lr=1e300), dict(grad_scale=1e39), dict(grad_scale=-1e300)):
        assert adamw(lib, wrong) == E, wrong
