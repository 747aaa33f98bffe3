"""8-bit moments over many steps: the rounding that hot_adamw_step trains with keeps them at the 64-bit ones on average.  On the definition that
the kernel is held to bit by bit."""
import ctypes as C
import inspect
import math

import numpy as np
import pytest

import paper_2503_21261_amd as hot
import moment_oracle as drawn
import tune_oracle as ref
from test_tune_ops_cpu import at, table, tensor

BETA1 = 0.9


def gradients(kind, n, steps, seed=0):
    rng = np.random.default_rng(seed)
    for t in range(steps):
        g = rng.standard_normal(n) * 1e-2
        if kind == "constant":
            g = np.full(n, 1e-2)
        elif kind == "none after a while":
            g = g if t < 500 else np.zeros(n)
        elif kind == "rare":
            g = g * (rng.random(n) < 0.02) * (1.0 if t < steps // 2 else 0.1)
        elif kind == "a tenth after a while":
            g = g * (1.0 if t < steps // 3 else 0.1)
        yield g


@pytest.mark.parametrize("beta2", [0.999, 0.9999, 0.95])
@pytest.mark.parametrize("kind", ["even", "constant", "none after a while", "rare", "a tenth after a while"])
def test_moments_follow_over_thousands_of_steps(kind, beta2):
    # Gradients that are all alike make elements at the same place of their block alike: one block of those.  With 0.95 and no gradients v
    # falls by half every 14 steps and is at its smallest code after some hundred.
    n, steps = (1024 if kind == "constant" else 4096), 600 if beta2 == 0.95 and kind == "none after a while" else 3000
    for held, exact, err in drawn.follow(drawn.steps(gradients(kind, n, steps), n, BETA1, beta2), BETA1, beta2):
        assert abs(held - exact) <= err, (held, exact, err)
    assert err <= 0.5 * exact               # of v: the bound says something


def test_roundings_without_draws_do_not_follow():
    """What the header says of the other two: right in one step, and no rounding to train with."""
    own = lambda m, v, seed: (ref.held_m(m, False), ref.held_v(v, False))
    nearest = lambda m, v, seed: (ref.held_m(m, True), ref.held_v(v, True))
    for kind, hold in (("none after a while", own), ("a tenth after a while", own), ("constant", own), ("none after a while", nearest)):
        _, (held, exact, err) = drawn.follow(drawn.steps(gradients(kind, 1024, 3000), 1024, BETA1, 0.999, hold=hold), BETA1, 0.999)
        assert abs(held - exact) > err, (kind, held / exact)


def test_draws_are_uniform_and_new_in_every_step():
    """Over 4096 steps: the numbers that decide have the mean and the variance of even ones at each of the eight places, and do not go with the step
    before (six standard deviations)."""
    n, steps = 1024, 4096
    rng = np.random.default_rng(1)
    m, v = (rng.standard_normal(n).astype(np.float32) for _ in range(2))
    v = v * v
    d = np.stack([drawn.draws(m, v, drawn.seed_of(1e-3, 0.9, 0.999, s)) for s in range(1, steps + 1)])
    for bits, size in ((d >> 12, 1 << 20), (d & 0xFFFF, 1 << 16)):
        x = (bits.astype(np.float64) + 0.5) / size - 0.5
        for place in range(8):
            y = x[:, place::8]                    # 128 numbers of a step
            assert abs(y.mean()) < 6 / math.sqrt(12 * y.size)
            assert abs((y * y).mean() - 1 / 12) < 6 * math.sqrt(1 / 180 / y.size)
        # an element's own: 1024 means of 4096 numbers, products with those of the step before
        assert np.abs(x.mean(0)).max() < 6 / math.sqrt(12 * steps)
        assert abs((x[1:] * x[:-1]).mean()) < 6 / 12 / math.sqrt(x.size / 8)


def test_rounding_is_right_on_average():
    rng = np.random.default_rng(2)
    m, v = rng.standard_normal(1024).astype(np.float32), (rng.standard_normal(1024) ** 2).astype(np.float32)
    steps, sum_m, sum_v = 4096, np.zeros(1024), np.zeros(1024)
    for s in range(1, steps + 1):
        cm, cv = drawn.held(m, v, drawn.seed_of(1e-3, 0.9, 0.999, s))
        sum_m += ref.read_m(*cm)
        sum_v += ref.read_v(*cv)
    step = np.exp2(cm[1].astype(np.float64) - 133).repeat(32)
    top = np.abs(m) > 127 * step                 # held at 127
    assert (np.abs(sum_m / steps - m)[~top] <= (6 / 2 / math.sqrt(steps) + 2.0 ** -17) * step[~top]).all()
    assert (np.abs(sum_v / steps - v) <= 6 / 2 / math.sqrt(steps) * v / 8).all()


def test_steps_have_seeds_of_their_own():
    """Also past the corrections' end (0.5^25 and 0.9^165 are less than half a unit of 1), where the step's number tells the steps apart; before
    it a recorded call's are an eager one's."""
    for beta1, beta2 in ((0.9, 0.999), (0.5, 0.9), (0.0, 0.0)):
        seeds = [drawn.seed_of(1e-3, beta1, beta2, s) for s in range(1, 20001)]
        assert len(set(seeds)) >= 19998           # of 2^32 numbers: 0.05 pairs by chance
    for s in range(1, 9000):
        assert drawn.seed_of(1e-3, 0.9, 0.999, s) == drawn.step_seed(1e-3, 1 - 0.9 ** s, 1 - 0.999 ** s)


def test_training_rounds_by_draws_and_unknown_ways_are_refused():
    assert inspect.signature(hot.hot_adamw_step).parameters["rounding"].default == hot.HOT_ROUND_DRAWN == 3
    st, t = table([tensor()])
    assert st == hot.HOT_OK
    for rounding, count in ((2, 0), (4, 0), (-1, 0), (3, 1), (3, 3), (3, 6), (3, -1), (1, 2)):
        cfg = hot.hot_adamw_config(1e-3, 0.9, 0.99, 1e-8, 1, rounding, count, at(0).value)
        assert hot.lib().hot_adamw_step(t, C.byref(cfg), None) == hot.HOT_ERR_ARG
    cfg = hot.Config(rounding=hot.HOT_ROUND_DRAWN)              # the linear backward has no steps to draw by
    assert hot.lib().hot_workspace_bytes(C.byref(cfg.c()), 64, 64, 64) == 0
