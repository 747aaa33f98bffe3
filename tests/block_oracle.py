"""Plain 64-bit forms of the operators around the linear backward, for the tests: numpy and torch on the CPU, written
from the formulas, without the library.  Every tolerance is returned beside its value, derived from the number of fp32 roundings
(u = 2^-24 each, relative) between the inputs and the output."""
import math

import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}      # rounding of a store, relative (fp32: counted with the others)


def f64(t):
    return t.detach().cpu().double()


# ---- 8-bit checkpoint: exact, codes and exponents as the layout holds them -----------------------------------------

def checkpoint_layout(rows, cols):
    pitch = (cols + 31) // 32 * 32
    exps = (rows * pitch + 255) // 256 * 256
    return pitch, exps, exps + rows * pitch // 32


def checkpoint(t):
    """(codes [rows, pitch] int8, exponents [rows, groups] uint8, values [rows, cols] float64) of a CPU tensor."""
    a = t.detach().cpu().float().numpy().astype(np.float64)
    rows, cols = a.shape
    pitch, _, _ = checkpoint_layout(rows, cols)
    whole = np.zeros((rows, pitch))
    whole[:, :cols] = a
    g = whole.reshape(rows, pitch // 32, 32)
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    top = np.abs(g).max(-1)
    e = np.full(top.shape, 8)
    for k in range(8, 255):         # the smallest step that leaves 127 or less after rounding
        e = np.where(np.rint(top * 2.0 ** (133 - e)) > 127, np.minimum(e + 1, 254), e)
    codes = np.clip(np.rint(g * 2.0 ** (133.0 - e)[..., None]), -127, 127)
    values = np.where(bad[..., None], np.nan, codes * 2.0 ** (e - 133.0)[..., None])
    e = np.where(bad, 255, e)
    return codes.reshape(rows, pitch).astype(np.int8), e.astype(np.uint8), torch.from_numpy(values.reshape(rows, pitch)[:, :cols])


# ---- activations ------------------------------------------------------------------------------------------------------

def _tail(x):
    """Phi(-|x|) and its absolute error in the kernels: a fit to 4e-7, a reciprocal and an exponential of one unit in the
    last place (2 u) each, three products, and x^2 / 2 rounded three times before it is an exponent."""
    tail = 0.5 * torch.special.erfc(x.abs() * math.sqrt(0.5))      # ndtr is 1 + erf, which cancels here
    return tail, tail * (5e-7 + 8 * U + 3 * U * 0.5 * x * x)


def _sigmoid(arg, roundings):
    """sigmoid(arg), 1 - sigmoid(arg), and the error of the first: the exponential, the sum and the reciprocal (6 u), and an argument off by
    `roundings` u, relative, whose effect is arg * (1 - sigmoid)."""
    s, r = torch.sigmoid(arg), torch.sigmoid(-arg)
    return s, r, s * (6 * U + roundings * U * arg.abs() * r) + 2.0 ** -126


def _tanh_arg(x):
    c = x.clamp(-30, 30)
    return 2 * math.sqrt(2 / math.pi) * (c + 0.044715 * c ** 3), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * c * c)


def act(fn, x):
    """(f(x), tolerance) for float64 x."""
    if fn == "none":
        return x, torch.zeros_like(x)
    if fn == "relu":
        return x.clamp(min=0), torch.zeros_like(x)
    if fn == "gelu":
        tail, d = _tail(x)
        y = torch.where(x > 0, x - x * tail, x * tail)
        return y, x.abs() * d + 3 * U * y.abs()
    arg, rounds = (_tanh_arg(x)[0], 8) if fn == "gelu_tanh" else (x, 3)
    s, _, d = _sigmoid(arg, rounds)
    return x * s, x.abs() * d + 2 * U * (x * s).abs()


def act_slope(fn, x):
    if fn == "none":
        return torch.ones_like(x), torch.zeros_like(x)
    if fn == "relu":
        return (x > 0).double(), torch.zeros_like(x)
    if fn == "gelu":
        tail, d = _tail(x)
        bell = torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi) * x
        return torch.where(x < 0, tail, 1 - tail) + bell, d + bell.abs() * (6 * U + 3 * U * 0.5 * x * x) + 4 * U
    if fn == "gelu_tanh":
        arg, up = _tanh_arg(x)
        s, r, d = _sigmoid(arg, 8)
        c = x.clamp(-30, 30)
        return s + c * s * r * up, d + (c * up).abs() * (d * r + s * (d + U) + 6 * U * s * r) + 2 * U
    s, r, d = _sigmoid(x, 3)
    return s * (1 + x * r), d * (1 + x.abs() * r) + s * x.abs() * (d + U) + 4 * U * (s * (1 + x.abs() * r))


def act_grad(fn, g_y, x, dtype):
    """(g_x, tolerance, sum over rows, its tolerance)."""
    slope, d = act_slope(fn, x)
    g, dg = g_y * slope, g_y.abs() * d + U * (g_y * slope).abs()
    # a column's sum: at most 128 additions one after the other at the sizes of the tests
    return g, dg + HALF[dtype] * (g.abs() + dg), g.sum(0), dg.sum(0) + 128 * U * g.abs().sum(0)


# ---- layer norm ---------------------------------------------------------------------------------------------------------

def norm(h, gamma, beta, eps, dtype):
    """y, mean, rstd of float64 h, each with its tolerance.  A lane adds at most 64 elements, ten more additions join the lanes:
    75 roundings of a sum; the mean is taken twice, so that only deviations are rounded."""
    cols = h.shape[1]
    mean = h.mean(1, keepdim=True)
    d = h - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    spread = d.abs().mean(1, keepdim=True)
    n = d * rstd
    g = gamma if gamma is not None else torch.ones(cols, dtype=torch.float64)
    b = beta if beta is not None else torch.zeros(cols, dtype=torch.float64)
    y = n * g + b
    # deviations are exact to u of |h - first mean|, which differs from |d| by 75 u mean|h|
    first = 75 * U * h.abs().mean(1, keepdim=True)
    dn = rstd * (3 * U * (d.abs() + first) + 80 * U * (spread + first)) + 80 * U * n.abs()
    dy = g.abs() * dn + 3 * U * ((n * g).abs() + b.abs())
    dmean = 2 * U * mean.abs() + 80 * U * (spread + first)
    return (y, dy + HALF[dtype] * (y.abs() + dy)), (mean[:, 0], dmean[:, 0]), (rstd[:, 0], 80 * U * rstd[:, 0])


def norm_grad(g_y, h, gamma, mean, rstd, g_residual, dtype):
    """(g_x, g_gamma, g_beta), each with its tolerance, from the mean and rstd that the forward call left."""
    cols = h.shape[1]
    mean, rstd = mean[:, None], rstd[:, None]
    n = (h - mean) * rstd
    t = g_y * (gamma if gamma is not None else torch.ones(cols, dtype=torch.float64))
    m1, m2 = t.mean(1, keepdim=True), (t * n).mean(1, keepdim=True)
    g = rstd * (t - m1 - n * m2)
    d1, d2 = 80 * U * t.abs().mean(1, keepdim=True), 84 * U * (t * n).abs().mean(1, keepdim=True)
    dg = rstd * (6 * U * t.abs() + d1 + 4 * U * m1.abs() + n.abs() * d2 + 8 * U * (n * m2).abs())
    if g_residual is not None:
        g = g + g_residual
        dg = dg + U * g.abs()
    gn = g_y * n
    return ((g, dg + HALF[dtype] * (g.abs() + dg)), (gn.sum(0), 132 * U * gn.abs().sum(0)), (g_y.sum(0), 128 * U * g_y.abs().sum(0)))


# ---- forward product -----------------------------------------------------------------------------------------------------

def product(x, w, bias):
    """x.w^T + bias of float64 operands and its tolerance: factors to 22 bits at least relative to their row's largest value (three
    such errors a product), at most I / 2 + 64 additions one after the other."""
    z = x @ w.t().contiguous()
    size = x.abs() @ w.abs().t().contiguous()
    top = x.abs().amax(1, keepdim=True), w.abs().amax(1, keepdim=True)
    tiny = 2.0 ** -38 * (top[0] * w.abs().sum(1)[None] + x.abs().sum(1, keepdim=True) * top[1].t())
    # no fp32 result is nearer than 2^-150, half the smallest fp32 number, however it was computed: a product and an addition for
    # each of the I terms, and the result itself, may each be off by that where they fall below 2^-126
    d = size * (3 * 2.0 ** -22 + (x.shape[1] / 2 + 64) * U) + tiny + (2 * x.shape[1] + 1) * 2.0 ** -150
    if bias is not None:
        z = z + bias
        d = d + U * z.abs()
    return z, d


def linear(x, w, bias, fn, residual, dtype):
    """(y, tolerance), (z, tolerance)."""
    z, dz = product(x, w, bias)
    y, dy = act(fn, z)
    dy = dy + 1.2 * dz          # no activation here is steeper than 1.13
    if residual is not None:
        y = y + residual
        dy = dy + U * y.abs()
    return (y, dy + U * y.abs() + HALF[dtype] * (y.abs() + dy)), (z, dz)
