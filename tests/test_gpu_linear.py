"""kavg_linear and kavg_linear_backward against 64 bits, element by element."""
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L

pytestmark = pytest.mark.gpu

DTYPES = (torch.float32, torch.bfloat16)
IDS = ("f32", "bf16")
CODE = dict(zip(L.ACTS, (kavg.KAVG_ACT_NONE, kavg.KAVG_ACT_RELU, kavg.KAVG_ACT_SILU)))
# sets, rows, inputs, outputs: single elements, tails of every kind of tile, contractions that are split
SIZES = [(1, 1, 1, 1), (2, 1, 8, 8), (3, 3, 5, 7), (1, 33, 64, 33), (2, 64, 64, 64), (1, 65, 130, 67), (2, 128, 128, 128), (1, 130, 72, 300), (1, 257, 264, 520),
         (1, 300, 1, 9), (2, 1, 1000, 3), (1, 17, 2000, 130), (3, 40, 4096, 24), (1, 2, 4099, 1030), (16, 1, 96, 640), (1, 5000, 24, 40), (1, 5001, 23, 41), (2, 2049, 63, 33),
         (2, 16, 1000, 100), (1, 15, 72, 8200), (3, 9, 4104, 1030), (2, 128, 1024, 10), (1, 5000, 264, 16), (3, 17, 520, 1), (1, 16640, 512, 5)]
# as many tiles of the largest kind as there are compute units
LARGE = [(4, 2048, 72, 2040), (4, 2047, 136, 2048), (1, 4096, 64, 4096)]


def normal(seed, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def apart(t, pad, first=0):
    """t as columns first .. of a tensor with longer rows, NaN around it."""
    whole = torch.full((*t.shape[:-1], t.shape[-1] + pad + first), float("nan"), dtype=t.dtype, device="cuda")
    whole[..., first:first + t.shape[-1]] = t
    return whole[..., first:first + t.shape[-1]]


def in_rows(w, turned, pad=0):
    """Weights [sets, outputs, inputs] in rows of a matrix of replicas, in either order, NaN behind them."""
    J, N, K = w.shape
    rows = torch.full((J, N * K + pad), float("nan"), dtype=w.dtype, device="cuda")
    at = rows[:, :N * K].view(J, K, N).transpose(1, 2) if turned else rows[:, :N * K].view(J, N, K)
    at.copy_(w)
    return at


def operands(size, dtype, seed=1):
    J, M, K, N = size
    return (normal(seed, J, M, K, dtype=dtype), normal(seed + 1, J, N, K, dtype=dtype, scale=K ** -0.5), normal(seed + 2, J, N, scale=0.3), normal(seed + 3, J, M, N, dtype=dtype))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES + LARGE, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
def test_forward(size, dtype, turned):
    x, w, b, residual = operands(size, dtype)
    at = in_rows(w, turned)
    for kind, bias, add, keep in (("none", None, None, False), ("relu", b, None, True), ("silu", b, residual, True)):
        got = kavg.kavg_linear(x, at, bias, activation=CODE[kind], residual=add, pre=keep)
        y, z = L.linear(x, w, bias, kind, add, dtype)
        L.close(got[0] if keep else got, y)
        if keep:
            L.close(got[1], z)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size", SIZES + LARGE, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
def test_backward(size, dtype, turned):
    x, w, _, dz = operands(size, dtype)
    pre = normal(9, *x.shape, dtype=dtype)
    at = in_rows(w, turned)
    for kind in L.ACTS:
        got = kavg.kavg_linear_backward(dz, x, at, activation=CODE[kind], pre=None if kind == "none" else pre)
        want = L.linear_backward(dz, x, w, kind, pre, dtype)
        for g, e in zip(got, want):
            L.close(g, e)
    assert got[1].stride(-1) == 1 or got[1].stride(-2) == 1
    # each gradient alone: the same bits
    for k in range(3):
        only = kavg.kavg_linear_backward(dz, x, at, activation=CODE[kind], pre=pre, out=None if k == 0 else False, dweight=None if k == 1 else False,
                                         dbias=None if k == 2 else False)
        assert [o is None for o in only] == [j != k for j in range(3)]
        assert torch.equal(only[k], got[k]) or k == 2
    L.close(only[2], want[2])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size,pad,first,step", [((2, 70, 64, 48), 8, 8, 16), ((2, 70, 64, 48), 3, 1, 5), ((3, 33, 31, 17), 2, 3, 1), ((1, 200, 100, 260), 12, 4, 0), ((2, 5, 40, 9), 1, 0, 3),
                                                 ((1, 64, 300, 8), 8, 0, 0)], ids=str)
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
def test_tensors_apart(size, pad, first, step, turned, dtype):
    """Everything lies in longer rows at any alignment; what lies between is read by no result and stays."""
    J, M, K, N = size
    x, w, b, residual = operands(size, dtype)
    pre, at = normal(9, *x.shape, dtype=dtype), in_rows(w, turned, step)

    def place(cols, dtype=dtype):
        whole = torch.full((J, M, cols + pad + first), 7.0, dtype=dtype, device="cuda")
        return whole, whole[..., first:first + cols]
    (y_all, y), (z_all, z), (dx_all, dx) = place(N), place(N), place(K)
    kavg.kavg_linear(apart(x, pad, first), at, apart(b, pad, first), activation=CODE["silu"], residual=apart(residual, pad, first), pre=z, out=y)
    want_y, want_z = L.linear(x, w, b, "silu", residual, dtype)
    L.close(y, want_y)
    L.close(z, want_z)
    flat = torch.full((J, N * K + N + step), 7.0, device="cuda")
    dw = flat[:, :N * K].view(J, K, N).transpose(1, 2) if turned else flat[:, :N * K].view(J, N, K)
    db = flat[:, N * K:N * K + N]
    kavg.kavg_linear_backward(apart(residual, pad, first), apart(x, pad, first), at, activation=CODE["silu"], pre=apart(pre, pad, first), out=dx, dweight=dw, dbias=db)
    for g, e in zip((dx, dw, db), L.linear_backward(residual, x, w, "silu", pre, dtype)):
        L.close(g, e)
    for whole, part in ((y_all, y), (z_all, z), (dx_all, dx)):
        part.fill_(7.0)
        assert (whole == 7.0).all()
    assert (flat[:, N * K + N:] == 7.0).all()
    # the gradient in the order that the weights do not have
    other = torch.empty(J, N, K, device="cuda") if turned else torch.empty(J, K, N, device="cuda").transpose(1, 2)
    kavg.kavg_linear_backward(residual, x, at, out=False, dweight=other, dbias=False)
    L.close(other, L.linear_backward(residual, x, w, "none", None, dtype)[1])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_learners_between_each_other_and_shared_operands(dtype):
    J, M, K, N = 3, 40, 48, 24
    x, w, b, r = operands((J, M, K, N), dtype)
    between = x.transpose(0, 1).contiguous().transpose(0, 1)              # [rows][sets][inputs]
    y = torch.empty(M, J, N, dtype=dtype, device="cuda").transpose(0, 1)
    kavg.kavg_linear(between, w, b, residual=r, out=y)
    assert torch.equal(y, kavg.kavg_linear(x, w, b, residual=r))
    one, same = w[:1].expand(J, N, K), x[:1].expand(J, M, K)
    assert torch.equal(kavg.kavg_linear(x, one, b[:1].expand(J, N)), kavg.kavg_linear(x, one.contiguous(), b[:1].repeat(J, 1)))
    row = r[:, :1].expand(J, M, N)
    assert torch.equal(kavg.kavg_linear(same, w, residual=row), kavg.kavg_linear(same.contiguous(), w, residual=row.contiguous()))
    for g, e in zip(kavg.kavg_linear_backward(row, same, one), kavg.kavg_linear_backward(row.contiguous(), same.contiguous(), one.contiguous())):
        assert torch.equal(g, e)
    flat = kavg.kavg_linear(x[0], w[0], b[0], residual=r[0])
    assert flat.shape == (M, N)
    L.close(flat, L.linear(x[0], w[0], b[0], "none", r[0], dtype)[0])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("size", [(2, 70, 64, 48), (1, 9, 2000, 33), (1, 1, 512, 256)], ids=str)
def test_in_place(size, dtype):
    """y is the residual; dx is pre, or x; results are those of other places, to the last bit, also a second time."""
    x, w, b, r = operands(size, dtype)
    pre = normal(9, *x.shape, dtype=dtype)
    want = kavg.kavg_linear(x, w, b, activation=CODE["silu"], residual=r)
    at = r.clone()
    assert kavg.kavg_linear(x, w, b, activation=CODE["silu"], residual=at, out=at) is at and torch.equal(at, want)
    dx, dw, db = kavg.kavg_linear_backward(r, x, w, activation=CODE["relu"], pre=pre)
    for over in (pre.clone(), x.clone()):
        given = dict(x=x, pre=over) if torch.equal(over, pre) else dict(x=over, pre=pre)
        got = kavg.kavg_linear_backward(r, given["x"], w, activation=CODE["relu"], pre=given["pre"], out=over)
        assert got[0] is over and torch.equal(over, dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_relu_takes_its_output_for_pre(dtype):
    x, w, _, dz = operands((2, 70, 64, 48), dtype)
    pre = normal(9, *x.shape, dtype=dtype)
    a, b = (kavg.kavg_linear_backward(dz, x, w, activation=CODE["relu"], pre=p)[0] for p in (pre, pre.clamp(min=0)))
    assert torch.equal(a, b) and (a[pre <= 0] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("turned", (False, True), ids=("", "turned"))
@pytest.mark.parametrize("size", [(1, 70, 100, 48), (1, 3, 1000, 64), (2, 200, 72, 264)], ids=str)
def test_infinities_and_nan_stay_in_their_rows_and_columns(size, turned, dtype):
    J, M, K, N = size
    x, w, b, dz = operands(size, dtype)
    clean = kavg.kavg_linear(x, in_rows(w, turned), b)
    clean_back = kavg.kavg_linear_backward(dz, x, in_rows(w, turned))
    x[0, M // 2, K - 1], w[0, N - 1, 0] = float("inf"), float("nan")
    y = kavg.kavg_linear(x, in_rows(w, turned), b)
    assert torch.isnan(y[0, :, N - 1]).all() and not torch.isfinite(y[0, M // 2]).any()
    keep = torch.ones(J, M, N, dtype=torch.bool, device="cuda")
    keep[0, M // 2], keep[0, :, N - 1] = False, False
    assert torch.equal(y[keep], clean[keep])
    dx, dw, db = kavg.kavg_linear_backward(dz, x, in_rows(w, turned))
    assert torch.isnan(dx[0, :, 0]).all() and torch.equal(dx[..., 1:], clean_back[0][..., 1:])
    assert not torch.isfinite(dw[0, :, K - 1]).any() and torch.equal(dw[..., :K - 1], clean_back[1][..., :K - 1]) and torch.equal(db, clean_back[2])
    dz[0, M - 1, 0] = float("-inf")
    dx, dw, db = kavg.kavg_linear_backward(dz, x, in_rows(w, turned))
    assert db[0, 0] == float("-inf") and torch.equal(db[0, 1:], clean_back[2][0, 1:])
    assert torch.equal(dx[0, :M - 1, 1:], clean_back[0][0, :M - 1, 1:]) and torch.equal(dw[0, 1:, :K - 1], clean_back[1][0, 1:, :K - 1])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_no_rows_and_no_learners(dtype):
    w = normal(1, 2, 5, 8, dtype=dtype)
    none = torch.empty(2, 0, 8, dtype=dtype, device="cuda")
    assert kavg.kavg_linear(none, w).shape == (2, 0, 5)
    dw, db = torch.full((2, 5, 8), 7.0, device="cuda"), torch.full((2, 5), 7.0, device="cuda")
    dx, _, _ = kavg.kavg_linear_backward(torch.empty(2, 0, 5, dtype=dtype, device="cuda"), none, w, dweight=dw, dbias=db)
    assert dx.shape == none.shape and (dw == 0).all() and (db == 0).all()
    assert kavg.kavg_linear_backward(torch.empty(2, 0, 5, dtype=dtype, device="cuda"), none, w, dweight=False)[2].eq(0).all()
    assert kavg.kavg_linear(torch.empty(0, 3, 8, dtype=dtype, device="cuda"), w[:0]).shape == (0, 3, 5)
    assert kavg.kavg_linear_backward(torch.empty(0, 3, 5, dtype=dtype, device="cuda"), torch.empty(0, 3, 8, dtype=dtype, device="cuda"), w[:0])[1].shape == (0, 5, 8)


def test_rows_past_32_bits():
    """Operands whose rows lie past 2^32 elements: bf16 rows of a wide tensor, one of them as the result."""
    wide = torch.empty(5, (1 << 30) + 8, dtype=torch.bfloat16, device="cuda")
    x = wide[:, :64]
    x.copy_(normal(1, 5, 64, dtype=torch.bfloat16))
    w = normal(2, 48, 64, dtype=torch.bfloat16)
    y = wide[:, 1 << 29:(1 << 29) + 48]
    kavg.kavg_linear(x, w, out=y)
    L.close(y, L.linear(x, w, None, "none", None, torch.bfloat16)[0])
    dx = wide[:, 1 << 30:(1 << 30) + 8]
    kavg.kavg_linear_backward(y, x[:, :8], w[:, :8], out=dx, dweight=False, dbias=False)
    L.close(dx, L.linear_backward(y, x[:, :8], w[:, :8], "none", None, torch.bfloat16)[0])
    dw = kavg.kavg_linear_backward(y, x, w, out=False)[1]
    L.close(dw, L.linear_backward(y, x, w, "none", None, torch.bfloat16)[1])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_on_a_side_stream_and_under_graphs(dtype):
    """Three graphs, replayed in turns with eager calls between them, on inputs that change."""
    sizes = [(2, 70, 2000, 48), (1, 200, 64, 72), (1, 4096, 64, 4096)]
    static = [operands(s, dtype) for s in sizes]
    graphs, outs = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = [t.clone().zero_() for t in static[0]]
        slow = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            slow = slow @ slow * 1e-2
        for t, s in zip(late, static[0]):
            t.copy_(s)
        y = kavg.kavg_linear(late[0], late[1], late[2], residual=late[3])
    side.synchronize()
    assert torch.equal(y, kavg.kavg_linear(static[0][0], static[0][1], static[0][2], residual=static[0][3]))

    def work(x, w, b, r):
        y, z = kavg.kavg_linear(x, w, b, activation=CODE["silu"], pre=True)
        return (y, z, *kavg.kavg_linear_backward(r, x, w, activation=CODE["silu"], pre=x))
    for s in static:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(work(*s))
        graphs.append(graph)
    for k in range(4):
        for j, s in enumerate(static):
            for t, n in zip(s, operands(sizes[j], dtype, seed=20 + 7 * k + j)):
                t.copy_(n)
        for j in (0, 1, 2) if k % 2 else (2, 1, 0):
            graphs[j].replay()
        torch.cuda.synchronize()
        for j, s in enumerate(static):
            assert all(torch.equal(a, b) for a, b in zip(outs[j], work(*s)))


def test_the_same_call_gives_the_same_bits():
    x, w, b, dz = operands((2, 300, 2000, 260), torch.bfloat16)
    first = (kavg.kavg_linear(x, w, b), *kavg.kavg_linear_backward(dz, x, w))
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, (kavg.kavg_linear(x, w, b), *kavg.kavg_linear_backward(dz, x, w))))


@pytest.mark.parametrize("kind", ("none", "silu"))
def test_gradients_are_differences(kind):
    """In fp32, a sum of the result's values times g against its change along a direction: a change of h = 2^-6 in the direction, forward and back, leaves
    an error of h^2/6 of the third derivative (SiLU's is below 1 in size, in units of the direction's values here below 1/4 each way) and the
    roundings of two sums of M N values over 2h."""
    M, K, N, h = 20, 24, 12, 2.0 ** -6
    x, w, b, g = normal(1, M, K) / 2, normal(2, N, K) / 4, normal(3, N), normal(4, M, N) / 8

    def f(x):
        a = x * torch.sigmoid(x) if kind == "silu" else x
        return float((kavg.kavg_linear(a.float(), w, b).double() * g.double()).sum())
    a = (x * torch.sigmoid(x)) if kind == "silu" else x
    dx, dw, db = kavg.kavg_linear_backward(g, a, w, activation=CODE[kind], pre=x if kind != "none" else None)
    for seed in range(3):
        d = normal(10 + seed, M, K) / 4
        slope = (f(x + h * d) - f(x - h * d)) / (2 * h)
        third = float((g.abs().double() @ w.abs().double() * d.abs().double() ** 3).sum())
        size = float((g.abs().double() * (a.abs().double() @ w.abs().double().t() + b.abs().double())).sum())
        assert abs(slope - float((dx.double() * d.double()).sum())) <= h * h / 6 * third + 2 * (K + 8) * L.U * size / h
    # linear in W and b: exact but for roundings
    dW, dB = normal(5, N, K), normal(6, N)
    change = float(((kavg.kavg_linear(a, w + dW, b + dB).double() - kavg.kavg_linear(a, w, b).double()) * g.double()).sum())
    size = float((g.abs().double() * (a.abs().double() @ (w.abs() + dW.abs()).double().t() * 2 + b.abs().double() + dB.abs().double())).sum())
    assert abs(change - float((dw.double() * dW.double()).sum() + (db.double() * dB.double()).sum())) <= 4 * (K + M * N) * L.U * size
