"""Numbers that no call takes are refused as such by the binding, whatever Python makes of them."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import lib  # noqa: F401  (the loaded library)


@pytest.fixture
def host_tensors(monkeypatch, lib):  # noqa: F811
    """The checks of the numbers come behind the one that x is a device tensor."""
    kavg._torch()
    monkeypatch.setattr(kavg, "_dtype", lambda x, name: kavg.KAVG_FP32)


@pytest.mark.parametrize("kw", [dict(eps=1e300), dict(eps=-1e300), dict(eps=None), dict(eps="1"), dict(seed=1.5), dict(seed=None), dict(seed=1 << 64),
                                dict(site=-1), dict(site=None), dict(drop="x"), dict(groups="2"), dict(groups=2.0), dict(activation=None)], ids=str)
def test_group_norm(host_tensors, kw):
    x = torch.zeros(2, 3, 8)
    with pytest.raises(kavg.KavgError) as e:
        kavg.kavg_group_norm(x, None, None, **dict(dict(groups=2), **kw))
    assert e.value.code == kavg.KAVG_EINVAL


@pytest.mark.parametrize("kw", [dict(seed=None), dict(seed="1"), dict(site=None), dict(seed=1 << 64), dict(seed=-1), dict(site=1 << 24)], ids=str)
def test_dropout(host_tensors, kw):
    for call in (kavg.kavg_dropout, kavg.kavg_dropout_backward):
        with pytest.raises(kavg.KavgError) as e:
            call(torch.zeros(2, 8), 0.5, **dict(dict(seed=1), **kw))
        assert e.value.code == kavg.KAVG_EINVAL
