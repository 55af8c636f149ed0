"""AdamW steps of the library: moments bit by bit, 8-bit states code by code, parameters within a bound of their 64-bit values."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L

pytestmark = pytest.mark.gpu

OPTIONS = dict(lr=2e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
LENGTHS = [1, 3, 4, 255, 256, 257, 1000, 1024, 2047, 2048, 2049, 5000, 70001]


def normal(seed, *shape, scale=1.0):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale


def away(p):
    """bf16 patterns of fp32 values, to nearest, ties away from zero."""
    bits = p.astype(np.float32).view(np.uint32)
    return ((bits + np.uint32(0x8000)) >> np.uint32(16)).astype(np.uint16)


def decoded(codes, scales, rows):
    table = np.concatenate([L.e4m3_values(), [np.nan]])
    c = codes.reshape(rows, -1)
    v = table[c & 0x7F] * np.where(c & 0x80, -1.0, 1.0)
    return (v * np.repeat(scales, L.BLOCK, 1)[:, :c.shape[1]]).astype(np.float32).reshape(codes.shape)


def host(t):
    return t.view(torch.uint8).cpu().numpy() if t.dtype is torch.float8_e4m3fn else t.detach().float().cpu().numpy() if t.dtype is torch.bfloat16 else t.detach().cpu().numpy()


def check_step(plan, grads, step, seed=0, options=OPTIONS, grad_scale=1.0, decays=None):
    """One step of the plan against the reference, from the plan's own present state."""
    before = [[host(t).copy() for t in (p, g, *s)] for p, g, s in zip(plan.params, grads, plan.states)]
    plan.step(grads, step, seed=seed, grad_scale=grad_scale, **(dict(options, weight_decay=decays) if decays else options))
    for i, ((p, g, *state), s) in enumerate(zip(before, plan.states)):
        rows = state[2].shape[0] if plan.bits == 8 else 1
        m, v = state[:2]
        if plan.bits == 8:
            m, root = decoded(m, state[2], rows), decoded(v, state[3], rows)
            v = root * root
        o = dict(options, weight_decay=decays[i] if decays else options["weight_decay"])
        (want, bound), m, v = L.adamw(p, g, m, v, step, grad_scale=grad_scale, **o)
        got = host(plan.params[i])
        off = np.abs(got - want)
        assert ((off <= bound) | (np.isnan(off) & np.isnan(want))).all(), (i, float(np.nanmax(off / bound)))
        if plan.bits == 32:
            assert np.array_equal(host(s[0]), m, equal_nan=True) and np.array_equal(host(s[1]), v, equal_nan=True)
        else:
            codes, scales = L.coded(m, rows)
            assert np.array_equal(host(s[2]), scales) and np.array_equal(host(s[0]).reshape(rows, -1), codes), i
            codes, scales = L.coded(np.sqrt(v), rows, L.draws(v.size, (seed + step) % (1 << 64), i))
            assert np.array_equal(host(s[3]), scales) and np.array_equal(host(s[1]).reshape(rows, -1), codes), i
        if plan.copies[i] is not None:
            assert np.array_equal(plan.copies[i].contiguous().view(torch.uint16).cpu().numpy(), away(got).reshape(got.shape))


def tensors(lengths, dtype, seed=1):
    params = [normal(seed + i, n, scale=0.1) for i, n in enumerate(lengths)]
    grads = [(normal(seed + 50 + i, n) * 1e-3 * torch.exp(2 * normal(seed + 90 + i, n))).to(dtype) for i, n in enumerate(lengths)]
    return params, grads


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("bits", (32, 8))
def test_many_lengths_at_once(bits, dtype):
    """Three steps from zero states; more tensors than a launch takes."""
    params, grads = tensors(LENGTHS * 3, dtype)
    copies = [torch.empty_like(p, dtype=torch.bfloat16) if i % 2 else None for i, p in enumerate(params)]
    plan = kavg.AdamW(params, bits=bits, copies=copies)
    for step in (1, 2, 1000):
        check_step(plan, grads, step, seed=(1 << 64) - 2, grad_scale=0.5 if step == 2 else 1.0)
        grads = [g.roll(1) for g in grads]


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("bits", (32, 8))
@pytest.mark.parametrize("shapes,pad", [(((7, 5), (5,), (300,), (33, 9)), 0), (((64, 64), (256,), (1,), (3, 1000)), 3), (((4096,),), 8)], ids=("small", "odd", "one"))
def test_learners_rows(shapes, pad, bits, dtype):
    """Parameters and copies in rows of the replicas, gradients in rows of their own and whole; what lies between stays."""
    P, sizes = 3, [int(np.prod(s)) for s in shapes]
    n = sum(sizes) + pad
    replicas, copies, grads_in = (torch.full((P, n), 7.0, device="cuda", dtype=t) for t in (torch.float32, torch.bfloat16, dtype))
    params, copy_of, grads, at = [], [], [], 0
    for i, (shape, size) in enumerate(zip(shapes, sizes)):
        a, b, g = (t[:, at:at + size].view(P, *shape) for t in (replicas, copies, grads_in))
        a.copy_(normal(i, P, *shape))
        g.copy_(normal(20 + i, P, *shape, scale=1e-2))
        params.append(a)
        copy_of.append(b)
        grads.append(g if i % 2 else g.contiguous())
        at += size
    plan = kavg.AdamW(params, bits=bits, copies=copy_of)
    for step in (1, 2):
        check_step(plan, grads, step, seed=5, decays=[0.0 if len(s) == 1 else 0.1 for s in shapes])
    assert (replicas[:, at:] == 7.0).all() and (copies[:, at:] == 7.0).all()


@pytest.mark.parametrize("first", (1, 2, 3))
@pytest.mark.parametrize("bits", (32, 8))
def test_any_start(bits, first):
    """Parameter, gradient, states and copy at any multiple of their elements."""
    n = 1500

    def at(t, k=first):
        whole = torch.zeros(n + 16, dtype=torch.uint8 if t is torch.float8_e4m3fn else t, device="cuda")
        return (whole.view(t) if t is torch.float8_e4m3fn else whole)[k:k + n], whole
    (p, p_all), (g, _), (c, c_all) = at(torch.float32), at(torch.bfloat16), at(torch.bfloat16)
    p.copy_(normal(1, n))
    g.copy_(normal(2, n, scale=1e-2).bfloat16())
    kept = [at(torch.float32 if bits == 32 else torch.float8_e4m3fn) for _ in "mv"]
    states = [s for s, _ in kept] + ([torch.full((1, 6), 2.0 ** -126, device="cuda") for _ in "mv"] if bits == 8 else [])
    plan = kavg.AdamW([p], states=[states], copies=[c])
    for step in (1, 2):
        check_step(plan, [g], step)
    for whole in (p_all, c_all, kept[0][1], kept[1][1]):
        assert (whole[:first] == 0).all() and (whole[first + n:] == 0).all()


@pytest.mark.parametrize("bits", (32, 8))
def test_extreme_values(bits):
    """Zeros, the smallest and largest magnitudes, infinities and NaN among ordinary gradients: each stays where it is."""
    p, g = normal(1, 2048), normal(2, 2048, scale=1e-2)
    g[256:512] = 0
    g[512:768] *= 1e-30
    g[768:1024] *= 1e20
    g[1024] = 3e38
    g[1280], g[1281], g[1282] = float("inf"), -float("inf"), float("nan")
    g[1536:1792] = float("nan")
    g[1800] = 1e-45
    plan = kavg.AdamW([p], bits=bits)
    for step in (1, 2, 3):
        check_step(plan, [g], step, options=dict(OPTIONS, eps=1e-6))
    bad = torch.isnan(plan.params[0])
    # (the square of 3e38 is infinite: a v of 32 bits stays so and stops its parameter, one of 8 bits has no infinity and is NaN from the second step on)
    assert bool(bad[1024]) == (bits == 8)
    bad[1024] = False
    assert bad[1280:1283].all() and bad[1536:1792].all() and not bad[:1280].any() and not bad[1283:1536].any() and not bad[1792:].any()


def test_codes_on_both_sides_of_every_value():
    """First steps whose moments, in units of their scales, are e4m3's values, the middles between them and the next fp32 values on both sides."""
    table = L.e4m3_values()
    table = table[table < 440]
    some = np.concatenate([table, (table[1:] + table[:-1]) / 2]).astype(np.float32)
    some = np.concatenate([np.nextafter(some, np.float32(0)), some, np.nextafter(some, np.float32(1e9))])
    some = some[some < 440]
    blocks = [np.concatenate([[440.0], part, np.zeros(255 - part.size)]) for part in np.array_split(some, -(-some.size // 255))]
    g = torch.from_numpy(np.concatenate(blocks).astype(np.float32)).cuda()
    for sign in (1, -1):
        # beta1 = 0: m is the gradient; beta2 = 0: the root is its magnitude
        plan = kavg.AdamW([torch.zeros_like(g)], bits=8)
        check_step(plan, [sign * g], 1, seed=3, options=dict(lr=1e-3, beta1=0.0, beta2=0.0, eps=1e-8, weight_decay=0.0))
        assert set(host(plan.states[0][0]).reshape(-1) & 0x7F) >= set(range(0x7E))


def test_rounding_of_roots_keeps_their_mean():
    """beta2 = 0.999 and gradients of 0: a root decays as it should on average, which rounded to nearest it could not (a step changes it by
    0.0005, half a unit is 0.03).  After 200 steps v is 0.999^200 of its start; the mean of 2^16 roots, each a random walk of at most 200 steps of variance
    below (1/8)^2 / 4 of its square, is off by less than five standard deviations."""
    n, steps = 1 << 16, 200
    plan = kavg.AdamW([torch.zeros(n, device="cuda")], bits=8)
    plan.step([torch.ones(n, device="cuda")], 1, beta2=0.999, seed=11)
    start = decoded(host(plan.states[0][1]), host(plan.states[0][3]), 1).astype(np.float64).mean()
    zero = torch.zeros(n, device="cuda")
    for step in range(2, 2 + steps):
        plan.step([zero], step, beta2=0.999, seed=11)
    got = decoded(host(plan.states[0][1]), host(plan.states[0][3]), 1).astype(np.float64).mean()
    want = start * 0.999 ** (steps / 2)
    assert abs(got - want) < 5 * want * (steps * 0.25 / 64 / n) ** 0.5 + 1e-6 * want


@pytest.mark.parametrize("bits", (32, 8))
def test_numbers_on_the_device_under_a_graph(bits):
    """Step, rate and factor read when the graph runs: replays are the eager steps of another plan, to the last bit; two graphs in turns."""
    rates, runs = [3e-3, 1e-3, 5e-4, 2e-3], []
    for k in range(2):
        params, grads = tensors([3000, 17, 256], torch.float32, seed=7 + k)
        eager = kavg.AdamW([p.clone() for p in params], bits=bits)
        plan = kavg.AdamW(params, bits=bits)
        step, lr, factor = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros((), device="cuda"), torch.ones(1, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.add_(1)
            plan.step(grads, step, lr=lr, grad_scale=factor, seed=40 + k, beta1=0.8, beta2=0.95)
        runs.append((plan, eager, grads, step, lr, factor, graph))
    for t, rate in enumerate(rates, 1):
        for k, (plan, eager, grads, step, lr, factor, graph) in enumerate(runs):
            lr.fill_(rate)
            factor.fill_(1 / t)
            for g in grads:
                g.mul_(-0.7)
            graph.replay()
            torch.cuda.synchronize()
            assert int(step) == t
            eager.step(grads, t, lr=float(np.float32(rate)), grad_scale=float(np.float32(1 / t)), seed=40 + k, beta1=0.8, beta2=0.95)
            for a, b in zip(plan.params + [s.view(torch.uint8) for st in plan.states for s in st], eager.params + [s.view(torch.uint8) for st in eager.states for s in st]):
                assert torch.equal(a, b)


def test_a_rate_on_the_device_with_a_step_of_the_host():
    params, grads = tensors([3000], torch.float32)
    one, two = (kavg.AdamW([p.clone() for p in params]) for _ in range(2))
    for t in (1, 2):
        one.step(grads, t, lr=torch.full((), 0.125, device="cuda"))
        two.step(grads, t, lr=0.125)
    assert torch.equal(one.params[0], two.params[0])


def test_streams_and_order():
    """A step on a side stream waits for what that stream holds; the same steps give the same bits."""
    params, grads = tensors([100000], torch.bfloat16)
    want = kavg.AdamW([p.clone() for p in params], bits=8)
    want.step(grads, 1, seed=1)
    late = [torch.zeros_like(g) for g in grads]
    plan = kavg.AdamW(params, bits=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        slow = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            slow = slow @ slow * 1e-2
        late[0].copy_(grads[0])
        plan.step(late, 1, seed=1)
    side.synchronize()
    assert torch.equal(plan.params[0], want.params[0])
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(plan.states[0], want.states[0]))


def test_rows_of_states_are_a_matter_of_their_scales():
    """A tensor without gaps can have states in rows; the parameters do not see it, and empty ones are left out."""
    p, g = normal(1, 6, 300), normal(2, 6, 300, scale=1e-2)
    for rows in (1, 2, 3, 6, 9):
        blocks = -(-1800 // rows // L.BLOCK)
        state = [torch.zeros(6, 300, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "mv"] + [torch.full((rows, blocks), 2.0 ** -126, device="cuda") for _ in "mv"]
        none = torch.empty(0, device="cuda")
        plan = kavg.AdamW([none, p.clone()], states=[kavg.AdamW.zeros(none, 8), state])
        for step in (1, 2):
            check_step(plan, [none, g], step, seed=9) if rows == 1 else plan.step([none, g], step, seed=9, **OPTIONS)
        if rows == 1:
            first = plan.params[1].clone()
        codes, scales = state[0], state[2]
        assert torch.equal(codes.float().view(rows, -1).abs().amax(1) > 220, torch.ones(rows, dtype=torch.bool, device="cuda")) and (scales > 2.0 ** -126).all()
    assert first.isfinite().all()


@pytest.mark.parametrize("bits", (32, 8))
def test_tensors_past_the_cache(bits):
    """A step of more bytes than the caches hold gives, for its first elements, the bits of a step of those alone."""
    n, some = 27_000_003, 100_000
    p, g = normal(1, n), normal(2, n, scale=1e-2).bfloat16()
    whole, part = kavg.AdamW([p.clone()], bits=bits), kavg.AdamW([p[:some].clone()], bits=bits)
    for step in (1, 2):
        whole.step([g], step, seed=3)
        part.step([g[:some].clone()], step, seed=3)
    ends = some if bits == 32 else some // L.BLOCK * L.BLOCK
    assert torch.equal(whole.params[0][:ends], part.params[0][:ends])
    for a, b in zip(whole.states[0], part.states[0]):
        k = ends if a.dim() == 1 else ends // L.BLOCK
        assert torch.equal(a.view(torch.uint8 if a.element_size() == 1 else a.dtype).reshape(-1)[:k], b.view(torch.uint8 if b.element_size() == 1 else b.dtype).reshape(-1)[:k])
    last = kavg.AdamW([p[-5:].clone()])
    last.step([g[-5:].clone()], 1)
    first = kavg.AdamW([p.clone()])
    first.step([g], 1)
    assert torch.equal(first.params[0][-5:], last.params[0])


def test_replicas_without_gaps_and_a_copy_in_wider_rows():
    """All parameters of all learners as one tensor, the copy in rows of whole eights, as the meta step's shadow."""
    p, g = normal(1, 3, 517), normal(2, 3, 517, scale=1e-2)
    shadow = torch.full((3, 520), 7.0, dtype=torch.bfloat16, device="cuda")
    plan = kavg.AdamW((t for t in [p]), copies=[shadow[:, :517]])
    for step in (1, 2):
        check_step(plan, [g], step)
    assert (shadow[:, 517:] == 7.0).all()


def test_refused_weight_decays_leave_those_of_before():
    params = [normal(80 + i, 70) for i in range(2)]
    before = [p.clone() for p in params]
    plan, grads = kavg.AdamW(params), [torch.zeros_like(p) for p in params]
    plan.step(grads, 1, weight_decay=0.0)
    for wrong in ([0.5, 1e300], [0.5], [0.5, None], 1e300):
        with pytest.raises(kavg.KavgError):
            plan.step(grads, 2, weight_decay=wrong)
        plan.step(grads, 2, weight_decay=0.0)
        # (zero gradients and moments: the change is 0 / eps, the decay's factor 1)
        assert all(torch.equal(p, b) for p, b in zip(params, before)), wrong
