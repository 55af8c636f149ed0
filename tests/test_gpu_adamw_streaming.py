"""AdamW steps whose tensors no cache holds: more bytes of a launch than 256 MB, counted as parameter, gradient and both states, take kernels of their own for every
width of a state and type of gradient; several rows, copies, odd ends and other tensors beside them."""
import numpy as np
import pytest
import torch

from paper_2110_00625_amd import kavg
from tests import learner_reference as L
from tests.test_gpu_adamw import OPTIONS, away, decoded, host, normal

pytestmark = pytest.mark.gpu

CACHE = 256_000_000


def check_columns(before, after, row, first, n, cols, bits, step, seed, site):
    """Columns first .. first + n (whole blocks, or up to the row's end) of a row against the definition.  before, after: (p, g, states.., copy) on the device,
    each [rows][..]."""
    cut = [host(t[row, first:first + n]) for t in (before[0], before[1], before[2], before[3])]
    p, g, m, v = cut
    at = first // L.BLOCK
    blocks = slice(at, at + -(-n // L.BLOCK))
    if bits == 8:
        m, root = (decoded(c, s[row, blocks].cpu().numpy()[None], 1) for c, s in ((m, before[4]), (v, before[5])))
        v = root * root
    (want, bound), m, v = L.adamw(p, g, m, v, step, **OPTIONS)
    got = host(after[0][row, first:first + n])
    assert (np.abs(got - want) <= bound).all(), (row, first)
    kept = [host(t[row, first:first + n]) for t in after[2:4]]
    if bits == 32:
        assert np.array_equal(kept[0], m) and np.array_equal(kept[1], v)
    else:
        e = row * cols + first
        # (the draws of these elements: those of the same numbers from a later start, in fours)
        drawn = L.draws(4 + n, seed + step + (e // 4) * 0x9E3779B97F4A7C15 & (1 << 64) - 1, site)[e % 4:][:n]
        for codes, scales, (want_codes, want_scales) in zip(kept, after[4:6], (L.coded(m, 1), L.coded(np.sqrt(v), 1, drawn))):
            assert np.array_equal(codes, want_codes[0]) and np.array_equal(scales[row, blocks].cpu().numpy(), want_scales[0]), (row, first)
    if after[-1] is not None:
        assert np.array_equal(after[-1][row, first:first + n].contiguous().view(torch.uint16).cpu().numpy(), away(got))


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("bits", (32, 8))
def test_rows_past_the_cache(bits, dtype):
    """Three learners' rows of replicas with a copy in rows of its own, and a tensor of a few values behind: first, last and middle columns of every row."""
    P, each = 3, 4 + (4 if dtype is torch.float32 else 2) + bits // 4
    cols = CACHE // each // P + 8192 + 3
    assert P * cols * each > CACHE
    replicas, shadow = torch.full((P, cols + 70), 7.0, device="cuda"), torch.full((P, cols + 72), 7.0, dtype=torch.bfloat16, device="cuda")
    params, copies = [replicas[:, :cols], replicas[:, cols:cols + 67]], [shadow[:, :cols], None]
    grads = [normal(5, P, cols, scale=1e-2).to(dtype), normal(6, P, 67, scale=1e-2).to(dtype)]
    for i, p in enumerate(params):
        p.copy_(normal(1 + i, P, p.shape[1], scale=0.1))
    plan = kavg.AdamW(params, bits=bits, copies=copies)
    for step in (1, 2):
        before = [[t.clone() for t in (p, g, *s)] for p, g, s in zip(params, grads, plan.states)]
        plan.step(grads, step, seed=21, **OPTIONS)
        for i, (p, g) in enumerate(zip(params, grads)):
            n = p.shape[1]
            after = (p, g, *plan.states[i], copies[i])
            tail = n // L.BLOCK * L.BLOCK
            # (a wavefront has four blocks under way, a workgroup sixteen)
            for first in {0, tail // 2 // L.BLOCK * L.BLOCK, max(tail - 17 * L.BLOCK, 0)}:
                for row in range(P):
                    check_columns(before[i], after, row, first, min(n - first, 24 * L.BLOCK), n, bits, step, 21, i)
        grads = [g.flip(1) for g in grads]
    assert (replicas[:, cols + 67:] == 7.0).all() and (shadow[:, cols:] == 7.0).all()


@pytest.mark.parametrize("dtype", (torch.float32, torch.bfloat16), ids=("f32", "bf16"))
@pytest.mark.parametrize("bits", (32, 8))
def test_the_same_bits_as_in_the_cache(bits, dtype):
    """The first elements' step is that of a plan of those alone, whose kernel is another."""
    each, some = 4 + (4 if dtype is torch.float32 else 2) + bits // 4, 400 * L.BLOCK
    n = CACHE // each + 5
    p, g = normal(1, n), normal(2, n, scale=1e-2).to(dtype)
    whole, part = kavg.AdamW([p.clone()], bits=bits), kavg.AdamW([p[:some].clone()], bits=bits)
    for step in (1, 2):
        whole.step([g], step, seed=3)
        part.step([g[:some].clone()], step, seed=3)
    assert torch.equal(whole.params[0][:some], part.params[0])
    for a, b in zip(whole.states[0], part.states[0]):
        a, b = (t.view(torch.uint8).reshape(-1) for t in (a, b))
        assert torch.equal(a[:b.numel()], b)


@pytest.mark.parametrize("rows", (1, 2, 3, 6, 9))
def test_a_first_step_does_not_see_the_rows_of_its_states(rows):
    """States of zeros are zeros in any number of rows: parameters after one step, which takes the moments before they are rounded, are the same to the last bit."""
    p, g = normal(1, 6, 300), normal(2, 6, 300, scale=1e-2)
    one = kavg.AdamW([p.clone()], bits=32)
    one.step([g], 1, seed=9, **OPTIONS)
    blocks = -(-1800 // rows // L.BLOCK)
    state = [torch.zeros(6, 300, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in "mv"] + [torch.full((rows, blocks), 2.0 ** -126, device="cuda") for _ in "mv"]
    plan = kavg.AdamW([p.clone()], states=[state])
    plan.step([g], 1, seed=9, **OPTIONS)
    assert torch.equal(plan.params[0], one.params[0])
