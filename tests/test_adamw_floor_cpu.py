"""What 8-bit states do to values far below their block's largest, on the CPU, with
the rounding that the update's own tests are written with.

v's least code is 2^-32 of a block's largest value at most, 2^-16 of a gradient;
m's is 2^-17 to 2^-18.  Below that v is mostly rounded to 0 where m now and then
is rounded up, and the next step divides by little more than eps.

The bound on a step with v kept above 0.  Gradients: the block's largest is G at
each step, the others are in [-rel G, rel G], rel at most 2^-14.  With m and v
divided by 1 - beta^t as the step does, their largest are G and G^2, so that the
least codes are u_m <= G 2^-16.8 (448 times the scale is at least the largest and
224 times it is less, and the least code is 2^-9) and u_v >= G^2 2^-31.8 (57344 and
2^-16).  |m| <= rel G + rounding errors, each of less than u_m and of mean 0, which
decay by beta1 a step: a variance of at most u_m^2 / 4 / (1 - beta1^2), six
deviations of which are 7 u_m.  With rel = 2^-14 = 7 * 2^-16.8 that is 14 u_m.
sqrt(v) >= 2^-15.9 G, halved for what the rounding of the largest v and its growth
from one step to the next move u_v by: 14 * 2^-16.8 / (2^-15.9 / 2) = 15 in units
of lr."""
import numpy as np
import pytest

import blockref as bref

LIMIT = 15.0
BETAS = [(0.9, 0.95), (0.9, 0.999)]
RELS = [2.0 ** -14, 2.0 ** -16, 2.0 ** -18, 2.0 ** -20]


def gradients(blocks, rel, steps, seed, noisy=True):
    """[steps][blocks * 128] in float32: each block's first is 1, the others at rel."""
    rng = np.random.default_rng(seed)
    for _ in range(steps):
        g = (rng.uniform(-1, 1, (blocks, 128)) if noisy else np.ones((blocks, 128))) * rel
        g[:, 0] = 1
        yield g.reshape(-1).astype(np.float32)


def two(codes):
    return np.repeat((codes.astype(np.uint32) << 23).view(np.float32), 128)


def value(codes, mant, emin, bias):
    """The magnitude that 8-bit codes stand for."""
    c = codes.astype(np.int64) & 0x7F
    e, f = c >> mant, (c & ((1 << mant) - 1)) / 2.0 ** mant
    return np.where(e == 0, f * 2.0 ** emin, (1 + f) * 2.0 ** (e - bias)).astype(np.float32)


def with_floor(codes, v):
    """A v above 0 has the least code at least."""
    return np.where((v > 0) & (codes == 0), np.uint8(1), codes)


def largest_step(grads, betas, floor, eps=1e-8, seed=3):
    """The largest single step of the small values, in units of lr."""
    worst, m, v = 0.0, None, None
    for t, g in enumerate(grads, 1):
        if m is None:
            m, v = np.zeros_like(g), np.zeros_like(g)
        m, v = bref.adamw_states(m, v, g, *betas)
        step = m / (1 - betas[0] ** t) / (np.sqrt(v.astype(np.float64) / (1 - betas[1] ** t)) + eps)
        worst = max(worst, float(np.abs(step.reshape(-1, 128)[:, 1:]).max()))
        r = bref.random_bits(0, len(g), t, seed)
        sm, sv = bref.block_scales(m, 8), bref.block_scales(v, 15)
        mc = bref.stochastic(m, sm, (r >> np.uint64(16)) << np.uint64(4), 3, -6, 7)
        vc = bref.stochastic(v, sv, (r & np.uint64(0xFFFF)) << np.uint64(5), 2, -14, 15)
        if floor:
            vc = with_floor(vc, v)
        m = value(mc, 3, -6, 7) * np.where(mc & 0x80, -1, 1).astype(np.float32) * two(sm)
        v = value(vc, 2, -14, 15) * two(sv)
    return worst


@pytest.mark.parametrize("noisy", [True, False])
@pytest.mark.parametrize("betas", BETAS)
@pytest.mark.parametrize("rel", RELS)
def test_a_step_is_bounded_where_v_is_kept(rel, betas, noisy):
    assert largest_step(gradients(8, rel, 400, 1, noisy), betas, True) <= LIMIT


@pytest.mark.parametrize("betas", BETAS)
def test_a_step_is_not_bounded_where_v_is_lost(betas):
    """Why: the same gradients, v rounded to 0 as often as its mean asks for."""
    assert largest_step(gradients(8, 2.0 ** -16, 400, 1), betas, False) > 5 * LIMIT


def test_the_flag_goes_with_8_bits_only():
    from test_block_cpu import G, INVALID, SCRATCH, adamw
    from paper_2607_16100_amd import llblock as lb

    for bits in (32 | lb.LL_ADAMW_FLOOR, lb.LL_ADAMW_FLOOR, 16 | lb.LL_ADAMW_FLOOR, 8 | 2 * lb.LL_ADAMW_FLOOR):
        assert adamw(bits=bits, m_scales=G, v_scales=G) == INVALID
    # (and with it the states' scales are needed as without)
    assert adamw(bits=8 | lb.LL_ADAMW_FLOOR) == INVALID
    assert adamw(bits=8 | lb.LL_ADAMW_FLOOR, m_scales=G, v_scales=G, work_bytes=63) == SCRATCH
