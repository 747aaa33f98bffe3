"""The drawn rounding of 8-bit moments as it is defined, operation by operation, and runs of steps in it and in 64 bits.  CPU only."""
import math

import numpy as np

import tune_oracle as ref

MASK = 0xFFFFFFFF


def mixed(x):
    """A bijection of 32 bits."""
    x = np.asarray(x, np.uint64) & MASK
    x = ((x ^ (x >> 16)) * 0x6A09E667) & MASK
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & MASK
    return x ^ (x >> 16)


def float_bits(x):
    return int(np.float32(x).view(np.uint32))


def step_seed(lr, c1, c2, word=0):
    """The seed of a step: of its learning rate, its corrections and a word of the caller's."""
    h = 0
    for x in (float_bits(lr), float_bits(c1), float_bits(c2), word):
        h = int(mixed(h ^ x ^ 0x9E3779B9))
    return h


def seed_of(lr, beta1, beta2, step):
    """That of a call with a step number: the number counts where the corrections are those of the step before."""
    c = [(np.float32(1.0 - beta1 ** s), np.float32(1.0 - beta2 ** s)) for s in (step, step - 1)]
    return step_seed(lr, *c[0], word=step if c[0] == c[1] else 0)


def draws(m, v, seed):
    """32 bits an element of whole blocks: one number of the seed and the eight's place in their block, evenly spread over the eight, shifted by
    the bits of what is rounded."""
    at = np.arange(len(m), dtype=np.uint64)
    h = mixed(seed + (at & 1023) // 8) + (at & 7) * 0x9E379E37
    return (h + m.view(np.uint32) + v.view(np.uint32)) & MASK


def held_m(t, draw):
    g = t.reshape(-1, 32)
    e = np.clip((np.abs(g).max(1).astype(np.float32).view(np.uint32) + 0x10000) >> 23, 8, 254).astype(np.int64)
    steps = g * ((260 - e) << 23).astype(np.uint32).view(np.float32)[:, None]
    part = ((draw & 0xFFFF).astype(np.float32) + np.float32(0.5)) * np.float32(2.0 ** -16)
    c = np.floor(steps + part.reshape(-1, 32))
    return np.clip(c, -127, 127).astype(np.int8).reshape(-1), e.astype(np.uint8)


def held_v(t, draw):
    b = t.reshape(-1, 32).view(np.uint32).astype(np.int64)
    k = (b + (draw >> 12).astype(np.int64).reshape(-1, 32)) >> 20
    e = np.clip((k >> 3).max(1), 32, 254)
    c = np.where(b == 0, 0, np.clip(k - ((e - 31) * 8)[:, None], 1, 255))
    return c.astype(np.uint8).reshape(-1), e.astype(np.uint8)


def held(m, v, seed):
    """(codes and exponents of m, codes and exponents of v)"""
    d = draws(m, v, seed)
    return held_m(m, d), held_v(v, d)


def steps(gradients, n, beta1, beta2, lr=1e-3, hold=held):
    """From nothing, after every gradient: the moments of n elements (whole blocks) before they are rounded, as they are held, and in 64 bits."""
    m = v = np.zeros(n, np.float32)
    mx = vx = np.zeros(n)
    for step, g in enumerate(gradients, 1):
        g = g.astype(np.float32)
        m2, v2 = ref.moments(m, v, g, beta1, beta2)
        cm, cv = hold(m2, v2, seed_of(lr, beta1, beta2, step))
        m, v = ref.read_m(*cm), ref.read_v(*cv)
        mx = beta1 * mx + (1 - beta1) * g.astype(np.float64)
        vx = beta2 * vx + (1 - beta2) * g.astype(np.float64) ** 2
        yield (m2, v2), (m, v), (mx, vx)


def follow(run, beta1, beta2):
    """(held, exact, how far apart they may be) of the sum of m and of the sum of v at the end of a run.

    A value between two neighbours lo and hi that goes to each with the other's distance for probability is right on average and has the variance
    (value - lo) (hi - value); what a step adds to it fades with beta^2 a step.  Eight neighbours, which share a number of the step, may go the
    same way: a sum has eight times the sum of the variances at most.  Six standard deviations; m above 127 steps of its group is held at
    127, which is half a step off at most; and u = 2^-24 three times a step, fading with beta."""
    var_m = var_v = 0.0
    for (m2, v2), (m, v), (mx, vx) in run:
        b = v2.view(np.uint32)
        lo, hi = (x.view(np.float32).astype(np.float64) for x in (b & np.uint32(0xFFF00000), (b & np.uint32(0xFFF00000)) + np.uint32(0x00100000)))
        var_v = beta2 ** 2 * var_v + float(((v2 - lo) * (hi - v2)).sum())
        e = np.clip((np.abs(m2).reshape(-1, 32).max(1).view(np.uint32) + 0x10000) >> 23, 8, 254).astype(np.int64)
        step = np.exp2((e - 133).astype(np.float64)).repeat(32)
        part = m2 / step - np.floor(m2 / step)
        var_m = beta1 ** 2 * var_m + float((part * (1 - part) * step ** 2).sum())
    u_m, u_v = (3 * ref.U / (1 - b) * float(np.abs(x).sum()) for b, x in ((beta1, mx), (beta2, vx)))
    return ((float(m.sum(dtype=np.float64)), float(mx.sum()), 6 * math.sqrt(8 * var_m) + float(step.sum()) / 2 + u_m),
            (float(v.sum(dtype=np.float64)), float(vx.sum()), 6 * math.sqrt(8 * var_v) + u_v))
