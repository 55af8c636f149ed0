"""What the layers refuse: at the C boundary before any device call (no GPU needed), and in the binding."""
import ctypes

import pytest
import torch

from paper_2110_00625_amd import kavg

NORM = dict(dtype=0, activation=0, sets=2, images=3, positions=4, channels=8, groups=2, eps=1e-5, reserved=0, drop=0.1, seed=1, site=0)
ORDER = ("dtype", "activation", "sets", "images", "positions", "channels", "groups", "eps", "reserved", "drop", "seed", "site")
AT = 4096                                    # an aligned address that no refused call reaches


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(kavg.LIB_PATH):
        from paper_2110_00625_amd import build
        build.build(verbose=False)
    return kavg.load_library()


def norm(**kw):
    d = dict(NORM, **kw)
    return kavg._NORM.pack(*[d[k] for k in ORDER])


def images(data=AT, sets=96, images_=32, row=8):
    return kavg._IMAGES.pack(data, sets, images_, row)


def forward(lib, n=None, x=None, y=None, w=AT, ws=8, b=AT, bs=8, mean=AT, rstd=AT):
    return lib.kavg_group_norm(norm() if n is None else n, images() if x is None else x, w, ws, b, bs, images() if y is None else y,
                               mean, rstd, AT, 1 << 30, None)


def backward(lib, n=None, dy=None, x=None, dx=None, mean=AT, rstd=AT, w=AT, ws=8, dw=AT, dws=8, db=AT, dbs=8):
    pick = lambda t: images() if t is None else t  # noqa: E731
    return lib.kavg_group_norm_backward(norm() if n is None else n, pick(dy), pick(x), mean, rstd, w, ws, AT, 8, pick(dx), dw, dws, db, dbs,
                                        AT, 1 << 30, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=-1), dict(activation=3), dict(activation=-1), dict(sets=-1), dict(images=-1), dict(positions=-1), dict(channels=0),
    dict(groups=0), dict(groups=3), dict(groups=-2), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
    dict(reserved=1), dict(drop=-0.1), dict(drop=1.1), dict(drop=float("nan")), dict(site=1 << 24), dict(sets=1 << 20, images=1 << 10, positions=1 << 10),
    dict(sets=1 << 62, images=1 << 62), dict(images=0, positions=1 << 42),
])
def test_descriptions_that_say_nothing(lib, kw):
    n, size = norm(**kw), ctypes.c_size_t(7)
    assert lib.kavg_group_norm_workspace(n, 0, ctypes.byref(size)) == kavg.KAVG_EINVAL and size.value == 7
    assert forward(lib, n) == kavg.KAVG_EINVAL
    assert backward(lib, n) == kavg.KAVG_EINVAL


def test_workspace_of_a_good_description(lib):
    for backward_ in (0, 1):
        for kw in ({}, dict(dtype=1), dict(images=0), dict(positions=1 << 20, channels=320, groups=32)):
            size = ctypes.c_size_t(1 << 60)
            assert lib.kavg_group_norm_workspace(norm(**kw), backward_, ctypes.byref(size)) == kavg.KAVG_OK and size.value < 1 << 32
    assert lib.kavg_group_norm_workspace(norm(), 0, None) == kavg.KAVG_EINVAL
    assert lib.kavg_group_norm_workspace(None, 0, ctypes.byref(size)) == kavg.KAVG_EINVAL


def test_workspaces_that_are_too_small(lib):
    """Found before anything is launched."""
    big = dict(sets=1, images=1, positions=1 << 20, channels=64, groups=8)
    x = images()
    for backward_ in (0, 1):
        size = ctypes.c_size_t(0)
        n = norm(**(big if backward_ == 0 else NORM))
        assert lib.kavg_group_norm_workspace(n, backward_, ctypes.byref(size)) == kavg.KAVG_OK and size.value > 0

        def call(block, nbytes):
            if backward_:
                return lib.kavg_group_norm_backward(n, x, x, AT, AT, AT, 8, AT, 8, x, AT, 8, AT, 8, block, nbytes, None)
            return lib.kavg_group_norm(n, kavg._IMAGES.pack(AT, 0, 0, 64), AT, 0, AT, 0, kavg._IMAGES.pack(AT, 0, 0, 64), AT, AT, block, nbytes, None)
        assert call(AT, size.value - 1) == kavg.KAVG_ENOMEM and call(None, 0) == kavg.KAVG_ENOMEM
        assert call(None, size.value) == kavg.KAVG_EINVAL and call(AT + 4, size.value) == kavg.KAVG_EINVAL


def test_operands_that_are_not_there(lib):
    E = kavg.KAVG_EINVAL
    for bad in (images(data=0), images(data=AT + 2), images(row=-8), images(images_=-32), images(sets=-96), images(row=1 << 50)):
        assert forward(lib, x=bad) == E and forward(lib, y=bad) == E
        assert backward(lib, x=bad) == E and backward(lib, dy=bad) == E and backward(lib, dx=bad) == E
    for overlapping in (images(row=7), images(row=0), images(images_=31), images(images_=0), images(sets=95)):
        assert forward(lib, y=overlapping) == E and backward(lib, dx=overlapping) == E
    assert forward(lib, mean=None) == E and forward(lib, rstd=None) == E
    assert backward(lib, mean=None) == E and backward(lib, rstd=None) == E
    assert forward(lib, w=AT + 1) == E and forward(lib, ws=-8) == E and forward(lib, bs=-1) == E
    assert backward(lib, dw=AT + 2) == E and backward(lib, dws=7) == E and backward(lib, dbs=0) == E and backward(lib, ws=-1) == E
    assert lib.kavg_group_norm(None, images(), AT, 8, AT, 8, images(), AT, AT, None, 0, None) == E
    assert lib.kavg_group_norm(norm(), None, AT, 8, AT, 8, images(), AT, AT, None, 0, None) == E


def test_dropout_refusals(lib):
    E = kavg.KAVG_EINVAL

    def drop(x=AT, xs=8, r=None, rs=0, y=AT, ys=8, rows=4, cols=8, dtype=0, p=0.5, seed=1, site=0):
        a = lib.kavg_dropout(x, xs, r, rs, y, ys, rows, cols, dtype, p, seed, site, None)
        if r is None:
            assert lib.kavg_dropout_backward(x, xs, y, ys, rows, cols, dtype, p, seed, site, None) == a
        return a
    for kw in (dict(x=None), dict(y=None), dict(x=AT + 1), dict(y=AT + 2), dict(r=AT + 3, rs=8), dict(r=AT, rs=-1), dict(xs=-1), dict(ys=7), dict(ys=-8),
               dict(rows=-1), dict(cols=0), dict(cols=-8), dict(dtype=2), dict(p=-0.01), dict(p=1.01), dict(p=float("nan")), dict(site=1 << 24),
               dict(rows=1 << 40, cols=1 << 40), dict(rows=1 << 39), dict(xs=1 << 60)):
        assert drop(**kw) == E, kw
    assert drop(rows=0) == kavg.KAVG_OK
    assert drop(rows=0, x=None, y=None) == kavg.KAVG_OK


def test_binding_wants_device_tensors(lib):
    x = torch.zeros(2, 3, 8)
    w = torch.ones(8)
    for call in (lambda: kavg.kavg_group_norm(x, w, w, 2), lambda: kavg.kavg_group_norm_backward(x, x, w, w, w, w, 2),
                 lambda: kavg.kavg_dropout(x, 0.5, 1), lambda: kavg.kavg_dropout_backward(x, 0.5, 1)):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == kavg.KAVG_EINVAL


@pytest.mark.gpu
def test_binding_refuses_what_does_not_fit(lib):
    d = "cuda"
    x, w, b = torch.zeros(2, 3, 5, 8, device=d), torch.ones(2, 8, device=d), torch.zeros(2, 8, device=d)
    _, mean, rstd = kavg.kavg_group_norm(x, w, b, 2, stats=True)
    f, g = kavg.kavg_group_norm, kavg.kavg_group_norm_backward
    nchw = torch.zeros(2, 3, 8, 5, device=d).transpose(2, 3)
    calls = [
        lambda: f(nchw, w, b, 2), lambda: f(x.half(), w, b, 2), lambda: f(x[0, 0], w[0], b[0], 2), lambda: f(x, w, b, 3), lambda: f(x, w, b, 0), lambda: f(x, w, b, -1, stats=True), lambda: f(x, w, b, 16, stats=True), lambda: f(x, w, b, None),
        lambda: f(x, w, b, 2, eps=0.0), lambda: f(x, w, b, 2, activation=9), lambda: f(x, w, b, 2, drop=1.5), lambda: f(x, w, b, 2, seed=-1),
        lambda: f(x, w, b, 2, site=1 << 24), lambda: f(x, w[0], b, 2), lambda: f(x, w.bfloat16(), b, 2), lambda: f(x, w.cpu(), b, 2),
        lambda: f(x, w.t().contiguous().t(), b, 2), lambda: f(x, w, b, 2, out=x.bfloat16()), lambda: f(x, w, b, 2, out=x[:1]),
        lambda: f(x, w, b, 2, out=x[:1].expand_as(x)), lambda: f(x, w, b, 2, out=nchw),
        lambda: g(x[:1], x, mean, rstd, w, b, 2), lambda: g(x, x, mean[:1], rstd, w, b, 2), lambda: g(x, x, mean.double(), rstd, w, b, 2),
        lambda: g(x, x, mean, rstd, w, b, 4), lambda: g(x, x, mean, rstd, w, b, 2, dweight=w[:1]), lambda: g(x, x, mean, rstd, w, b, 2, dbias=w[:1].expand(2, 8)),
        lambda: kavg.kavg_dropout(x.half(), 0.5, 1), lambda: kavg.kavg_dropout(x, 0.5, -1), lambda: kavg.kavg_dropout(x, 0.5, 1 << 64),
        lambda: kavg.kavg_dropout(x, 2.0, 1), lambda: kavg.kavg_dropout(x, 0.5, 1, residual=x[:1]), lambda: kavg.kavg_dropout(nchw, 0.5, 1),
        lambda: kavg.kavg_dropout(x, 0.5, 1, out=x[:1].expand_as(x)), lambda: kavg.kavg_dropout(torch.zeros(3, 4, 8, device=d)[:, ::3], 0.5, 1),
    ]
    for k, call in enumerate(calls):
        with pytest.raises(kavg.KavgError) as e:
            call()
        assert e.value.code == kavg.KAVG_EINVAL, k
