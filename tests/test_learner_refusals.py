"""What the products and the AdamW step refuse: at the C boundary before any device call (no GPU needed), and in the binding."""
import ctypes

import pytest
import torch

from paper_2110_00625_amd import kavg
from tests.test_layers_refusals import AT, lib  # noqa: F401  (lib: the loaded library)

E, OK = kavg.KAVG_EINVAL, kavg.KAVG_OK
MOST, COLUMNS = (1 << 31) - (1 << 16), 1 << 27
AWAY = 1 << 20                               # another address that no refused call reaches


def product(dtype=0, activation=0, sets=2, rows=4, inputs=8, outputs=6):
    return kavg._PRODUCT.pack(dtype, activation, sets, rows, inputs, outputs)


def rows(data=AT, sets=32, row=8):
    return kavg._MATRIX.pack(data, sets, row)


def weights(data=2 * AT, sets=48, o=8, i=1):
    return kavg._WEIGHTS.pack(data, sets, o, i)


def forward(lib, p=None, x=rows(), w=weights(), b=AT, bs=6, r=None, y=rows(AWAY), pre=None, block=AWAY, nbytes=0):  # noqa: F811
    return lib.kavg_linear(product() if p is None else p, x, w, b, bs, r, y, pre, block, nbytes, None)


def backward(lib, p=None, dz=rows(), x=rows(3 * AT), w=weights(), pre=None, dx=rows(AWAY), dw=weights(2 * AWAY), db=AT, dbs=6, block=AWAY, nbytes=0):  # noqa: F811
    return lib.kavg_linear_backward(product() if p is None else p, dz, x, w, pre, dx, dw, db, dbs, block, nbytes, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=-1), dict(activation=3), dict(activation=-1), dict(sets=-1), dict(rows=-1), dict(inputs=0), dict(outputs=0), dict(inputs=-8),
    dict(rows=MOST + 1), dict(inputs=COLUMNS + 1), dict(outputs=COLUMNS + 1), dict(sets=1 << 31), dict(sets=1 << 62), dict(sets=1, rows=1 << 30, inputs=1 << 12),
    dict(sets=1 << 12, rows=1, inputs=1 << 15, outputs=1 << 15), dict(sets=0, rows=1 << 30, outputs=1 << 12),
])
def test_descriptions_that_say_nothing(lib, kw):  # noqa: F811
    p, size = product(**kw), ctypes.c_size_t(7)
    assert lib.kavg_linear_workspace(p, 0, ctypes.byref(size)) == E and size.value == 7
    assert forward(lib, p) == E and backward(lib, p) == E


def test_workspaces(lib):  # noqa: F811
    size = ctypes.c_size_t(0)
    assert lib.kavg_linear_workspace(product(), 0, None) == E and lib.kavg_linear_workspace(None, 0, ctypes.byref(size)) == E
    for kw in (dict(sets=0), dict(rows=0), dict(dtype=1, sets=1, rows=MOST, inputs=8, outputs=8), dict(sets=1, rows=8, inputs=COLUMNS, outputs=8),
               dict(sets=1, rows=1, inputs=1, outputs=COLUMNS), dict(sets=(1 << 31) - 1, rows=1, inputs=8, outputs=1)):
        for back in (0, 1):
            assert lib.kavg_linear_workspace(product(**kw), back, ctypes.byref(size)) == OK and size.value < 1 << 40, kw
    # one row of results from a long contraction: split, and refused before a launch without the block
    long = dict(sets=1, rows=64, inputs=1 << 20, outputs=64)
    x, w, y = rows(row=1 << 20), weights(o=1 << 20), rows(AWAY, row=64)
    assert lib.kavg_linear_workspace(product(**long), 0, ctypes.byref(size)) == OK and size.value > 0
    p = product(**long)
    assert forward(lib, p, x=x, w=w, y=y, nbytes=size.value - 1) == kavg.KAVG_ENOMEM and forward(lib, p, x=x, w=w, y=y, block=None) == kavg.KAVG_ENOMEM
    assert forward(lib, p, x=x, w=w, y=y, block=None, nbytes=size.value) == E and forward(lib, p, x=x, w=w, y=y, block=AWAY + 4, nbytes=size.value) == E


def test_operands_that_are_not_there(lib):  # noqa: F811
    slope = product(activation=2)
    for bad in (rows(0), rows(AT + 2), rows(row=-8), rows(sets=-1), rows(row=1 << 50), rows(sets=1 << 50)):
        assert forward(lib, x=bad) == E and forward(lib, y=bad) == E and forward(lib, r=bad) == E and forward(lib, pre=bad) == E
        assert backward(lib, dz=bad) == E and backward(lib, x=bad) == E and backward(lib, dx=bad) == E and backward(lib, slope, pre=bad) == E
    for bad in (weights(0), weights(AT + 1), weights(i=2), weights(o=2, i=8), weights(o=-8), weights(sets=-1), weights(o=1 << 50), weights(o=1, i=1 << 50)):
        assert forward(lib, w=bad) == E and backward(lib, w=bad) == E and backward(lib, dw=bad) == E
    for overlapping in (rows(AWAY, row=5), rows(AWAY, row=0), rows(AWAY, sets=23, row=6), rows(AWAY, sets=0), rows(AWAY, sets=6, row=11)):
        assert forward(lib, y=overlapping) == E and forward(lib, pre=overlapping) == E
    for overlapping in (rows(AWAY, row=7), rows(AWAY, sets=0), rows(AWAY, sets=31)):
        assert backward(lib, dx=overlapping) == E
    for overlapping in (weights(2 * AWAY, sets=47), weights(2 * AWAY, o=7), weights(2 * AWAY, o=1, i=5), weights(2 * AWAY, sets=0)):
        assert backward(lib, dw=overlapping) == E
    assert forward(lib, b=AT + 2) == E and forward(lib, bs=-1) == E and backward(lib, db=AT + 2) == E and backward(lib, dbs=5) == E
    assert forward(lib, x=None) == E and forward(lib, w=None) == E and forward(lib, y=None) == E and lib.kavg_linear(None, rows(), weights(), None, 0, None, rows(AWAY), None, None, 0, None) == E
    assert backward(lib, dz=None) == E and backward(lib, x=None) == E and backward(lib, w=None) == E and backward(lib, slope, pre=None) == E


def test_results_over_operands(lib):  # noqa: F811
    assert forward(lib, x=rows(AWAY)) == E and forward(lib, w=weights(AWAY)) == E and forward(lib, pre=rows(AWAY)) == E and forward(lib, pre=rows(AT)) == E
    assert forward(lib, pre=rows(2 * AT)) == E and forward(lib, r=rows(3 * AT), pre=rows(3 * AT)) == E and forward(lib, r=rows(AWAY, row=16)) == E
    assert backward(lib, dz=rows(AWAY)) == E and backward(lib, w=weights(AWAY)) == E and backward(lib, product(activation=1), pre=rows(AWAY, row=16)) == E


def test_nothing_to_do(lib):  # noqa: F811
    none = product(sets=0)
    assert forward(lib, none, x=rows(0), w=weights(0), y=rows(0)) == OK and backward(lib, none, dz=rows(0), x=rows(0), w=weights(0), dx=rows(0), dw=weights(0)) == OK
    assert forward(lib, product(rows=0), x=rows(0), y=rows(0)) == OK
    assert backward(lib, dz=rows(), dx=None, dw=None, db=None) == OK


# ---- AdamW ----------------------------------------------------------------------------------------------------------

TENSOR = dict(param=AT, grad=2 * AT, m=3 * AT, v=4 * AT, m_scale=0, v_scale=0, copy=0, rows=0, cols=5, param_stride=5, grad_stride=5, copy_stride=0, weight_decay=0.0, reserved=0)
STEP = dict(bits=32, grad_dtype=0, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, seed=0, step_dev=0, lr_dev=0, grad_scale_dev=0)


def adamw(lib, options=None, count=1, **kw):  # noqa: F811
    d = dict(TENSOR, **kw)
    table = ctypes.create_string_buffer(kavg._TENSOR.pack(*d.values()))
    return lib.kavg_adamw(kavg._STEP.pack(*dict(STEP, **(options or {})).values()), ctypes.addressof(table), count, None)


def test_adamw_refusals(lib):  # noqa: F811
    inf, nan = float("inf"), float("nan")
    assert adamw(lib) == OK                                  # (no rows: nothing to launch)
    for o in (dict(bits=16), dict(grad_dtype=2), dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(eps=-1e-8), dict(eps=inf),
              dict(grad_scale=nan), dict(step=0), dict(step_dev=AT + 4), dict(lr_dev=AT + 2), dict(grad_scale_dev=AT + 1)):
        assert adamw(lib, o) == E, o
    assert adamw(lib, count=-1) == E and lib.kavg_adamw(None, None, 0, None) == E
    options = kavg._STEP.pack(*STEP.values())
    assert lib.kavg_adamw(options, None, 0, None) == OK and lib.kavg_adamw(options, None, 1, None) == E
    assert adamw(lib, dict(step=0, step_dev=AT)) == OK
    for kw in (dict(rows=-1), dict(cols=-1), dict(reserved=1), dict(weight_decay=-1.0), dict(weight_decay=nan)):
        assert adamw(lib, **kw) == E, kw
    for kw in (dict(rows=1 << 31), dict(rows=1 << 20, cols=1 << 20), dict(param=0), dict(grad=0), dict(m=0), dict(v=0), dict(m_scale=AT), dict(v_scale=AT), dict(param=AT + 2), dict(grad=AT + 2),
               dict(m=AT + 1), dict(v=AT + 2), dict(copy=AT + 1, copy_stride=5), dict(param_stride=4), dict(param_stride=1 << 46), dict(grad_stride=-1), dict(copy=AT, copy_stride=4)):
        assert adamw(lib, **dict(dict(rows=3), **kw)) == E, kw
    for kw in (dict(), dict(m_scale=AT), dict(v_scale=AT), dict(m_scale=AT, v_scale=AT + 2)):
        assert adamw(lib, dict(bits=8), **dict(dict(rows=3), **kw)) == E, kw


def test_binding_wants_device_tensors(lib):  # noqa: F811
    x, w = torch.zeros(3, 8), torch.ones(5, 8)
    for call in (lambda: kavg.kavg_linear(x, w), lambda: kavg.kavg_linear_backward(torch.zeros(3, 5), x, w), lambda: kavg.AdamW([w]), lambda: kavg.AdamW([w], bits=8), lambda: kavg.AdamW([w], bits=4),
                 lambda: kavg.kavg_linear(x, None)):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == E


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit(lib):  # noqa: F811
    d = "cuda"
    x, w, b, y = torch.zeros(2, 5, 8, device=d), torch.ones(2, 6, 8, device=d), torch.zeros(2, 6, device=d), torch.zeros(2, 5, 6, device=d)
    f, g = kavg.kavg_linear, kavg.kavg_linear_backward
    every_other = torch.zeros(2, 6, 16, device=d)[:, :, ::2]
    calls = [
        lambda: f(x.half(), w.half()), lambda: f(x, w.bfloat16()), lambda: f(x[0], w), lambda: f(x, w[0]), lambda: f(x, w[:1]), lambda: f(x[..., :7], w), lambda: f(x[0, 0], w[0, 0]),
        lambda: f(x.transpose(1, 2).contiguous().transpose(1, 2), w), lambda: f(x, every_other), lambda: f(x, w, b[:1]), lambda: f(x, w, b.bfloat16()), lambda: f(x, w, b.t().contiguous().t()),
        lambda: f(x, w, residual=y[:1]), lambda: f(x, w, residual=y.bfloat16()), lambda: f(x, w, out=y[:1].expand(2, 5, 6)), lambda: f(x, w, out=y.cpu()), lambda: f(x, w, activation=7),
        lambda: f(x, w, activation=None), lambda: f(x, w, pre=y[:1]), lambda: f(x, w, out=y, pre=y), lambda: f(x, w.cpu()),
        lambda: g(y[:1], x, w), lambda: g(y.bfloat16(), x, w), lambda: g(y, x, w, activation=1), lambda: g(y, x, w, activation=1, pre=y), lambda: g(y, x, w, out=x[:1].expand(2, 5, 8)),
        lambda: g(y, x, w, dweight=w[:1]), lambda: g(y, x, w, dweight=w.bfloat16()), lambda: g(y, x, w, dweight=every_other), lambda: g(y, x, w, dbias=b[:1].expand(2, 6)), lambda: g(y, x, w, dbias=b[0]),
    ]
    p, q = torch.zeros(3, 300, device=d), torch.zeros(7, device=d)
    A = kavg.AdamW
    eight = A.zeros(p, 8)
    calls += [
        lambda: A([p.bfloat16()]), lambda: A([p, p]), lambda: A([p], copies=[p]), lambda: A([p], copies=[]), lambda: A([p], states=[]), lambda: A([p], states=[(p,)]), lambda: A([p], states=[(q, q)]),
        lambda: A([p], states=[(p.clone(), p)]), lambda: A([p], states=[(p.clone(), p.clone().bfloat16())]), lambda: A([p, q], states=[A.zeros(p, 8), A.zeros(q, 32)]),
        lambda: A([p], states=[(*eight[:2], eight[2][:, :1], eight[3])]), lambda: A([p], states=[(*eight[:2], eight[2][:, :1].contiguous(), eight[3][:, :1].contiguous())]),
        lambda: A([p], states=[(*eight[:2], *(torch.ones(7, 1, device=d) for _ in "mv"))]), lambda: A([torch.zeros(4, 6, 8, device=d)[:, ::2, ::2]]),
        lambda: A([torch.zeros(4, 5, 6, device=d)[:, :3, :5]], bits=8), lambda: A([p.clone()[:1].expand(3, 300)]).step([p], 1),
        lambda: A([p]).step([], 1), lambda: A([p]).step([q], 1), lambda: A([p, q]).step([p.clone(), q.clone().bfloat16()], 1), lambda: A([p]).step([p.half()], 1), lambda: A([p]).step([p.clone()], 0),
        lambda: A([p]).step([p.clone()], 1, weight_decay=[0.1, 0.1]), lambda: A([p]).step([p.clone()], 1, beta1=1.0), lambda: A([p]).step([p.clone()], torch.ones(1, device=d)),
        lambda: A([p]).step([p.clone()], torch.ones(1, dtype=torch.int64)), lambda: A([p]).step([p.clone()], 1, lr=torch.ones(2, device=d)), lambda: A([p]).step([p.clone()], 1, seed=-1),
        lambda: A([p]).step([None], 1),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == E, k


def test_backward_that_has_a_block_for_its_first_product_alone(lib):  # noqa: F811
    # dW = dz^T x over 64 rows is not split, dx = dz W over 8192 outputs is: refused before either is launched (without a GPU the launch would say so)
    p = product(sets=1, rows=64, inputs=64, outputs=8192)
    size = ctypes.c_size_t(0)
    assert lib.kavg_linear_workspace(p, 1, ctypes.byref(size)) == OK and size.value > 0
    dz, x, w, dx, dw = rows(row=8192), rows(3 * AT, row=64), weights(o=64), rows(AWAY, row=64), weights(2 * AWAY, o=64)
    for block, nbytes, rc in ((AWAY, size.value - 1, kavg.KAVG_ENOMEM), (AWAY, 0, kavg.KAVG_ENOMEM), (None, 0, kavg.KAVG_ENOMEM), (None, size.value, E), (AWAY + 4, size.value, E)):
        assert backward(lib, p, dz=dz, x=x, w=w, dx=dx, dw=dw, block=block, nbytes=nbytes) == rc
