"""What training with the 8-bit moments of include/warp.h does over thousands of steps, beside 32-bit moments: a
simulation of the definition, which the GPU tests hold the kernel to code by code. The bounds are the statements
that the header and the design make about the format, its faults among them."""
from __future__ import annotations

import numpy as np
import pytest

F = np.float32


def cutoffs(levels, power):
    t = (np.arange(1, levels + 1, dtype=F) - F(0.5)) * F(1 / levels)
    t = t * t
    return t * t if power == 4 else t


CUT = {2: cutoffs(127, 2), 4: cutoffs(255, 4)}


def value(codes, top, power):
    t = np.abs(codes).astype(F) * F(1 / len(CUT[power]))
    t = t * t
    t = t * t if power == 4 else t
    return np.where(codes < 0, -t, t) * top


def coded(x, power):
    """Codes and scales of fp32 moments [blocks, 256]."""
    top = np.maximum(np.abs(x).max(1, keepdims=True), F(2.0 ** -126))
    share = np.abs(x) * (F(1) / top)
    codes = np.searchsorted(CUT[power], share.ravel(), side="right").reshape(x.shape)
    if power == 4:
        codes = np.maximum(codes, x > 0)
    return np.where(x < 0, -codes, codes), top


class Adam:
    """Steps in units of lr, of blocks of 256 elements, with moments in 8 or 32 bits."""

    def __init__(self, bits, blocks=4, beta1=0.9, beta2=0.999):
        self.bits, self.beta1, self.beta2, self.t = bits, beta1, beta2, 0
        self.m, self.v = np.zeros((2, blocks, 256), F)
        self.at = np.zeros((blocks, 256))

    def step(self, g):
        g = g.astype(F)
        self.t += 1
        m = self.m * F(self.beta1) + g * F(1 - self.beta1)
        v = self.v * F(self.beta2) + g * g * F(1 - self.beta2)
        self.at -= m / (1 - self.beta1 ** self.t) / (np.sqrt(v.astype(float) / (1 - self.beta2 ** self.t)) + 1e-8)
        if self.bits == 8:
            m, v = value(*coded(m, 2), 2), value(*coded(v, 4), 4)
        self.m, self.v = m, v

    def root(self):
        return np.sqrt(self.v.astype(float) / (1 - self.beta2 ** self.t))


HALF = np.arange(256) < 128


def spread(rng):
    return 10 ** rng.uniform(-3, 0, (4, 256))


def test_codes_that_rest():
    """Without a gradient, and with the block's largest kept, a first moment stays at its code up to code 9, and a
    second moment at every code."""
    for power, levels, beta, rests in ((2, 127, 0.9, 9), (4, 255, 0.999, 254)):
        codes = np.arange(levels + 1)
        x = value(codes, F(1), power) * F(beta)
        x[-1] = 1  # the block's largest
        blocks = np.pad(x, (0, 256 - len(x)))[None] if len(x) < 256 else x[None]
        after = coded(blocks.astype(F), power)[0][0, :levels + 1]
        moved = after != codes
        moved[-1] = False
        assert np.flatnonzero(moved).tolist() == list(range(rests + 1, levels))


def test_smallest_second_moment():
    """Code 1 is above zero while the scale is at least 2^-117: (1 / 255)^4 is 2^-31.98, the smallest number 2^-149."""
    assert value(np.array([1]), F(2.0 ** -117), 4)[0] > 0 and value(np.array([1]), F(2.0 ** -119), 4)[0] == 0
    assert coded(np.pad([F(2.0 ** -117), F(2.0 ** -149)], (0, 254))[None], 4)[0][0, 1] == 1


def test_steady_gradients():
    """Gradients whose spread varies by 1,000 inside a block: the root of v stays near it."""
    rng = np.random.default_rng(0)
    sigma, a = spread(rng), Adam(8)
    for _ in range(3000):
        a.step(sigma * rng.standard_normal(sigma.shape))
    low, high = np.quantile(a.root() / sigma, [0.05, 0.95])
    assert low > 0.7 and high < 1.3


@pytest.mark.parametrize("factor", [2, 4, 0.1])
def test_noisy_gradients_that_change(factor):
    """Half of a block's gradients change by a factor and the others do not: growth is followed, a fall is not while the
    block's largest stays, and steps stay too small."""
    sigma = spread(np.random.default_rng(0))
    runs = {}
    for bits in (8, 32):
        rng, a = np.random.default_rng(1), Adam(bits)
        for t in range(3500):
            now = np.where(HALF & (t >= 1500), sigma * factor, sigma)
            a.step(now * rng.standard_normal(now.shape))
        runs[bits] = np.quantile((a.root() / now)[:, HALF], [0.05, 0.5, 0.95])
    low, middle, high = runs[8]
    if factor > 1:
        assert low > 0.65 and high < 1.3
    else:
        assert middle > 1.5 * runs[32][1] and middle > 6


@pytest.mark.parametrize("factor", [2, 0.1])
def test_constant_gradients_that_change(factor):
    """Without noise a change of one step is (1 - beta2) (factor^2 - 1) of v, here at most 0.4%, and half a code at
    least 0.78%: under a largest that stays, the codes of gradients that double or fall tenfold stay what they were."""
    sigma = spread(np.random.default_rng(0))
    sigma[:, 255] = 2  # the largest, also when others have doubled
    a, exact = Adam(8), Adam(32)
    for t in range(3500):
        now = np.where(HALF & (t >= 1500), sigma * factor, sigma)
        a.step(now)
        exact.step(now)
        if t == 1499:
            before = coded(a.v, 4)[0]
    assert (coded(a.v, 4)[0] == before).all()
    assert (np.abs(exact.root() / now - 1)[:, HALF] < (0.1 if factor > 1 else 4)).all()


@pytest.mark.parametrize("noise,share,least,most", [(True, 1, 0.2, 0.6), (True, 0.1, 2, 5), (True, 0.005, 50, 120),
                                                    (False, 1, 8, 12), (False, 0.1, 80, 120)])
def test_gradients_that_vanish(noise, share, least, most):
    """Half of a block's gradients, `share` as large as the others, stop at step 500 and the others go on. From 100
    steps later on (32-bit moments have come to rest) the stopped elements go on moving, by this many lr in 2,400 steps."""
    drift = {}
    for bits in (8, 32):
        rng, a = np.random.default_rng(0), Adam(bits)
        for t in range(3000):
            g = rng.standard_normal((4, 256)) if noise else np.ones((4, 256))
            a.step(np.where(HALF, share * g if t < 500 else 0, g))
            if t == 599:
                then = a.at.copy()
        drift[bits] = np.median(np.abs(a.at - then)[:, HALF])
    assert drift[32] < 1e-3 and least < drift[8] < most


def test_gradients_that_turn():
    """A gradient that turns and is smaller than what a code's rest hides: m keeps the wrong sign, and the parameter
    moves the wrong way, as long as the block's largest stays. 32-bit moments turn with it. (Their steps: 0.0005 over a
    root that falls from 0.05 by exp(-t / 2000), 33 lr in all; those of 8 bits at least 0.003 / 0.05 each, 114 lr.)"""
    ends = {}
    for bits in (8, 32):
        a = Adam(bits, blocks=1)
        for t in range(3000):
            a.step(np.where(HALF, 0.05 if t < 1000 else -0.0005, 1.0)[None])
            if t == 1099:
                then = a.at.copy()
        ends[bits] = a.m[0, 0], (a.at - then)[0, 0]
    assert ends[32][0] == pytest.approx(-0.0005, rel=1e-3) and 25 < ends[32][1] < 45
    assert ends[8][0] > 0.003 and ends[8][1] < -100
