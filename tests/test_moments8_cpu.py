"""8-bit moments over thousands of updates, as their formats and their rounding are defined: they follow the recurrence of
AdamW.  (That the kernel's codes are these is tested on the GPU.)"""
import ctypes

import numpy as np
import pytest

from paper_2601_04342_amd import binding
from tests import moments8

F = np.float32


def run(kind, steps, marks, random=True, nearest_steps=8, betas=(0.9, 0.999), n=2048, seed=0):
    """{t: (mean and median of v / exact v, rms of the update / exact rms, median of m / exact m)}."""
    rng, (b1, b2) = np.random.default_rng(seed), betas
    codes = moments8.encode(np.zeros(n, F), np.zeros(n, F))
    M, V, out = np.zeros(n), np.zeros(n), {}
    for t in range(1, steps + 1):
        g = {"normal": lambda: rng.normal(size=n) * 1e-3, "constant": lambda: np.full(n, 1e-3),
             "around": lambda: 1e-3 * (1 + 0.3 * rng.normal(size=n)),
             "fall": lambda: rng.normal(size=n) * (1e-3 if t <= 1000 else 1e-4)}[kind]().astype(F)
        m, v = moments8.decode(*codes)
        m, v = F(b1) * m.astype(F) + F(1 - b1) * g, F(b2) * v.astype(F) + F(1 - b2) * (g * g)
        M, V = b1 * M + (1 - b1) * g.astype(float), b2 * V + (1 - b2) * g.astype(float)**2
        bits = moments8.random_bits(t, np.arange(n)) if random and t > nearest_steps else None
        codes = moments8.encode(m, v, bits)
        if t in marks:
            dm, dv = moments8.decode(*codes)
            rms = lambda m, v: np.sqrt(np.mean((m / (1 - b1**t) / (np.sqrt(v / (1 - b2**t)) + 1e-8))**2))
            out[t] = (dv / V).mean(), np.median(dv / V), rms(m, v) / rms(M, V), np.median(dm / M)
    return out


# What rounding at random may do.  A step of v's codes is s = 1/16 to 1/8 of v, 0.087 in the mean over the logarithm.  An
# update that changes v by (1 - b2) |g^2 / v - 1| v adds (1 - b2) |g^2 / v - 1| s v^2 of variance, of which the decay takes
# 2 (1 - b2) away: s / 2 times a mean of at most one = 0.044 stays, 0.21 v.  The mean of n = 2,048 is then known to 0.5 %
# (bound: four times that), the median to that, half a step of the codes, and half the variance; the update's rms rises
# by half the variance, 2.2 % (bound: twice that, and sampling).
MEAN, MEDIAN, RMS = 0.02, 0.005 + 1 / 16 + 0.022, 0.05


@pytest.mark.parametrize("kind", ["normal", "constant", "around"])
def test_moments_follow_adamw(kind):
    for t, (mean, median, rms, m) in run(kind, 3000, (30, 100, 1000, 3000)).items():
        assert abs(mean - 1) <= MEAN + (0.01 if t == 30 else 0), (kind, t)   # (an update is 1/30 of v then: half a step is not less)
        assert abs(median - 1) <= MEDIAN and abs(rms - 1) <= RMS, (kind, t)
        assert abs(m - 1) <= 1 / 16 + 0.01, (kind, t)      # half a step, beside which no mean is shifted


def test_moments_fall_with_the_gradients():
    """While v falls nothing takes the variance away: s for each of the time constants it falls through, less what the new
    gradients already are of it: 0.087 x 2.7 after three of them, 12 % of the rms; from there on it shrinks."""
    got = run("fall", 6000, (2000, 4000, 6000))
    for t, (mean, _, rms, _) in got.items():
        assert abs(mean - 1) <= 4 * 0.5 / np.sqrt(2048), t
        assert abs(rms - 1) <= (0.15 if t < 6000 else 0.1), t


def test_rounding_to_nearest_does_not():
    """What the rounding at random is for."""
    got = run("normal", 1000, (1000,), random=False)[1000]
    assert got[0] < 0.4 and got[2] > 1.5


def test_random_bits_are_spread():
    """Means, and products of neighbours in place and step, of 2^16 samples; a mean of uniform numbers is off by 1/sqrt(12 n)
    = 0.0011, a correlation by 0.004: bounds of five times that."""
    n = 1 << 16
    for step in (1, 9, 1000, 2**33 + 5):
        a = moments8.random_bits(step, np.arange(n))
        b = moments8.random_bits(step + 1, np.arange(n))
        for part in (lambda x: (x & np.uint64(0xFFFF)) / 2**16, lambda x: (x >> np.uint64(12)) / 2**20):
            x, y = part(a), part(b)
            assert abs(x.mean() - 0.5) <= 0.0056
            for u, w in ((x, y), (x[:-1], x[1:]), (x[:-32], x[32:]), (x[:-1024], x[1024:])):
                assert abs(np.corrcoef(u, w)[0, 1]) <= 0.02
    steps = np.array([moments8.random_bits(t, [77])[0] for t in range(20000)])
    for part in (lambda x: (x & np.uint64(0xFFFF)) / 2**16, lambda x: (x >> np.uint64(12)) / 2**20):
        x = part(steps)
        assert abs(x.mean() - 0.5) <= 0.0102 and abs(np.corrcoef(x[:-1], x[1:])[0, 1]) <= 0.036
    far = moments8.random_bits(9, np.arange(64, dtype=np.uint64) + np.uint64(2**34))
    assert (far != moments8.random_bits(9, np.arange(64))).sum() > 60


def test_a_negative_count_of_nearest_steps_is_refused():
    plan = binding.AdamWPlan(0x1000, 5, 2, 8)
    h = binding.AdamWHyper(1e-3, 0.9, 0.999, 1e-8, 0.01, None, -1)
    assert binding.library().rehyat_adamw_step(ctypes.byref(plan), ctypes.byref(h), None) == binding.E_SHAPE


def test_gradients_of_many_sizes_in_a_group():
    """Down to 2^-15 of the largest (v spans 30 binades) updates are AdamW's; below that v is held up by its least code and they
    shrink.  No m that is rounded up from next to nothing, to 2^-17 of the largest, meets a smaller divisor than 2^-15."""
    n, (b1, b2), rng = 1024, (0.9, 0.999), np.random.default_rng(1)
    spread = 2.0**-(np.arange(n) % 32)
    codes = moments8.encode(np.zeros(n, F), np.zeros(n, F))
    M, V, squares = np.zeros(n), np.zeros(n), np.zeros((2, 32))
    for t in range(1, 1001):
        g = (rng.normal(size=n) * 1e-3 * spread).astype(F)
        m, v = moments8.decode(*codes)
        m, v = F(b1) * m.astype(F) + F(1 - b1) * g, F(b2) * v.astype(F) + F(1 - b2) * (g * g)
        M, V = b1 * M + (1 - b1) * g.astype(float), b2 * V + (1 - b2) * g.astype(float)**2
        codes = moments8.encode(m, v, moments8.random_bits(t, np.arange(n)) if t > 8 else None)
        mine, exact = (a / (1 - b1**t) / np.sqrt(b / (1 - b2**t)) for a, b in ((m, v), (M, V)))
        # (after 8 updates to the nearest: an update of 1 is the first one's, 7.3 the most that AdamW makes of any gradients)
        assert np.abs(mine).max() <= 1.25 * max(1.0, np.abs(exact).max()), t
        if t > 500:
            squares += [(x * x).reshape(-1, 32).mean(0) for x in (mine, exact)]
    rms = np.sqrt(squares[0] / squares[1])
    assert (np.abs(rms[:15] - 1) <= RMS).all() and (rms[15:] <= 1 + RMS).all()
