"""What kavg.AdamW does with the tensors that it is given, without a GPU: the launch is replaced by one that writes down what it is handed."""
import gc

import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import lib  # noqa: F401  (the loaded library)


@pytest.fixture
def launched(lib, monkeypatch):  # noqa: F811
    """Tables of the launches, as tuples of their fields."""
    kavg._torch()
    tables = []

    def launch(x, fn, options, table, count):
        import ctypes
        size = kavg._TENSOR.size
        tables.append([kavg._TENSOR.unpack(ctypes.string_at(table + i * size, size)) for i in range(count)])
        return kavg.KAVG_OK
    monkeypatch.setattr(kavg, "_dtype", lambda x, name: kavg._DTYPES[x.dtype])
    monkeypatch.setattr(kavg, "_launch", launch)
    return tables


def refused(call):
    with pytest.raises(kavg.KavgError) as e:
        call()
    assert e.value.code == kavg.KAVG_EINVAL


def other_memory(p):
    p.data = torch.zeros_like(p)


def module_to(p):
    p.data = p.data.double()


def emptied(p):
    p.untyped_storage().resize_(0)


def grown(p):
    p.resize_(100000)


@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("move", (other_memory, module_to, emptied, grown))
def test_moved_parameters_and_copies_are_refused(launched, move, bits):
    for which in range(4):
        params = [torch.nn.Parameter(torch.ones(3, 70)) if i else torch.ones(5) for i in range(2)]
        copies = [None, torch.zeros(3, 70, dtype=torch.bfloat16)]
        plan, grads = kavg.AdamW(params, bits=bits, copies=copies if which < 3 else None), [torch.zeros(5), torch.zeros(3, 70)]
        plan.step(grads, 1)
        with torch.no_grad():
            move(copies[1] if which == 2 else params[which % 2].requires_grad_(False))
        done = len(launched)
        refused(lambda: plan.step(grads, 2))
        assert len(launched) == done


def test_other_entries_of_the_lists_are_refused(launched):
    params = [torch.ones(7), torch.ones(9)]
    for change in (lambda plan: plan.params.__setitem__(1, torch.ones(9)), lambda plan: plan.params.append(torch.ones(3)), lambda plan: plan.copies.__setitem__(0, None),
                   lambda plan: plan.params.__setitem__(0, None), lambda plan: plan.params.pop()):
        plan = kavg.AdamW(params, copies=[torch.zeros(7, dtype=torch.bfloat16), None])
        change(plan)
        refused(lambda: plan.step([torch.zeros_like(p) if p is not None else None for p in plan.params], 1))
    assert not launched


@pytest.mark.parametrize("bits", (32, 8))
def test_states_are_written_where_they_were(launched, bits):
    """States that are let go of, or whose tensors get other memory, stay allocated; `states` shows what is written."""
    p = torch.ones(3, 300)
    given = [list(kavg.AdamW.zeros(p, bits))]
    plan = kavg.AdamW([p], states=given)
    assert [s.data_ptr() for s in plan.states[0]] == [s.data_ptr() for s in given[0]]
    mine = given[0][0]
    mine.data = torch.zeros_like(mine)
    del given
    gc.collect()
    plan.states[0][1].data = torch.empty(0)
    plan.step([torch.zeros_like(p)], 1)
    assert list(launched[-1][0][2:4 if bits == 32 else 6]) == [s.data_ptr() for s in plan.states[0]]
    assert plan.states[0][1].shape == p.shape and mine.data_ptr() != plan.states[0][0].data_ptr()


def test_a_step_is_a_change_of_its_tensors_for_autograd(launched):
    """A graph that saved a parameter, a view of one, what it is a view of, or a copy, refuses its backward pass after a step, as after any change in place."""
    def of(kind):
        whole = torch.ones(3, 40)
        view = whole[:, 4:24].view(3, 4, 5)
        p = {"parameter": torch.nn.Parameter(torch.ones(3, 20)), "view": view, "base": view, "view of a view": view[:, 1:3], "detached": view.detach(), "copy": torch.ones(3, 20)}[kind]
        copy = torch.ones(3, 20, dtype=torch.bfloat16)
        return p, copy, {"base": whole, "copy": copy}.get(kind, p)
    for kind in ("parameter", "view", "base", "view of a view", "detached", "copy"):
        p, copy, saved = of(kind)
        plan = kavg.AdamW([p], copies=[copy] if kind == "copy" else None)
        x = torch.ones(saved.shape, dtype=saved.dtype, requires_grad=True)
        before, graph = saved._version, (x * saved.detach()).sum()
        plan.step([torch.zeros(p.shape)], 1)
        assert saved._version > before, kind
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            graph.backward()
        plan.step([torch.zeros(p.shape)], 2)
        (x * saved.detach()).sum().backward()
    with torch.inference_mode():
        p = torch.ones(5)
        kavg.AdamW([p]).step([torch.zeros(5)], 1)
    plan = kavg.AdamW([torch.ones(5)])
    version = plan.params[0]._version
    refused(lambda: plan.step([torch.zeros(6)], 1))
    assert plan.params[0]._version == version


@pytest.mark.parametrize("wrong", (None, 0.0, [0.0] * 7))
def test_what_is_no_gradient_is_refused_wherever_it_stands(launched, wrong):
    params = [torch.ones(7), torch.ones(7), torch.ones(7)]
    plan = kavg.AdamW(params)
    for i in (1, 2):
        refused(lambda: plan.step([wrong if k == i else torch.zeros(7) for k in range(3)], 1))
    assert not launched


def test_gradients_change_between_rows_and_whole_tensors(launched):
    """The table has the strides of this step's gradients, whatever those of the last were, also after a refused one."""
    params, rows = [torch.ones(3, 8)[:, :7], torch.ones(5)], torch.zeros(3, 11)[:, 2:9]
    plan = kavg.AdamW(params)
    for given in (torch.zeros(3, 7), rows, torch.zeros(3, 7), rows, torch.zeros(3, 9)[:, :7]):
        plan.step([given, torch.zeros(5)], 1)
        assert [t[1] for t in launched[-1]][0] == given.data_ptr() and [t[10] for t in launched[-1]] == [given.stride(0), 5]
        refused(lambda: plan.step([rows, None], 1))
