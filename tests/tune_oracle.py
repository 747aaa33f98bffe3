"""64-bit forms of the operators of a fine-tuning step, and the bounds that follow from fp32 arithmetic (u = 2^-24 for each operation,
relative) between the inputs and the output.  CPU only."""
import math

import numpy as np
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}     # half a step, relative


def owners(L, offsets, index, adapters):
    """Adapter of every row (-1: none) and whether the row belongs to a request."""
    if offsets is None:
        return torch.zeros(L, dtype=torch.int64), torch.ones(L, dtype=torch.bool)
    k, inside = torch.full((L,), -1, dtype=torch.int64), torch.zeros(L, dtype=torch.bool)
    for s in range(len(index)):
        lo, hi = int(offsets[s]), int(offsets[s + 1])
        inside[lo:hi] = True
        k[lo:hi] = int(index[s]) if 0 <= int(index[s]) < adapters else -1
    return k, inside


def adapter(x, a, b, scale, base, k, inside, y0, u0, g_y=None, g_base=None, g_x0=None):
    """{name: (value, largest error)} of a pass, all in 64 bits; y0, u0 and g_x0: what the outputs held before."""
    t, small = x.dtype, x.dtype == torch.bfloat16
    x, a, b = x.double(), a.double(), b.double()
    (L, I), (K, r, _), O = x.shape, a.shape, b.shape[1]
    s = torch.ones(K, dtype=torch.float64) if scale is None else scale.double()
    half = HALF[t]
    u, u_err = torch.zeros(L, r, dtype=torch.float64), torch.zeros(L, r, dtype=torch.float64)
    y = torch.zeros(L, O, dtype=torch.float64) if base is None else base.double().clone()
    y_err = torch.zeros(L, O, dtype=torch.float64)
    out = {}
    if g_y is not None:
        g_y = g_y.double()
        g_x = torch.zeros(L, I, dtype=torch.float64) if g_base is None else g_base.double().clone()
        g_x_err = torch.zeros(L, I, dtype=torch.float64)
        g_a, g_b = torch.zeros(K, r, I, dtype=torch.float64), torch.zeros(K, O, r, dtype=torch.float64)
        g_a_err, g_b_err = torch.zeros_like(g_a), torch.zeros_like(g_b)
    # A number enters a product with 16 bits or more where the result is bfloat16, whole otherwise.
    cut = 2.0 ** -16 if small else 0.0
    for j in range(K):
        rows = torch.nonzero(k == j)[:, 0]
        xr = x[rows]
        u[rows] = xr @ a[j].T
        u_err[rows] = (I + 4) * U * (xr.abs() @ a[j].abs().T)
        y[rows] += s[j] * (u[rows] @ b[j].T)
        whole = s[j].abs() * (u[rows].abs() @ b[j].abs().T)
        y_err[rows] = s[j].abs() * (u_err[rows] @ b[j].abs().T) + ((r + 4) * U + cut) * whole
        if g_y is None:
            continue
        g = g_y[rows]
        p = g @ b[j]
        p_err = (O + 4) * U * (g.abs() @ b[j].abs())
        g_x[rows] += s[j] * (p @ a[j])
        g_x_err[rows] = s[j].abs() * (p_err @ a[j].abs() + ((r + 4) * U + cut) * (p.abs() @ a[j].abs()))
        n = len(rows)
        g_a[j] = s[j] * (p.T @ xr)
        g_a_err[j] = s[j].abs() * (p_err.T @ xr.abs() + (n + 8) * U * (p.abs().T @ xr.abs()))
        g_b[j] = s[j] * (g.T @ u[rows])
        g_b_err[j] = s[j].abs() * (g.abs().T @ u_err[rows] + (n + 8) * U * (g.abs().T @ u[rows].abs()))
    y_err += 2 * U * y.abs() + half * (y.abs() + y_err)
    y[~inside], y_err[~inside] = y0.double()[~inside], 0.0
    u[~inside], u_err[~inside] = u0.double()[~inside], 0.0
    out.update(y=(y, y_err), u=(u, u_err))
    if g_y is not None:
        g_x_err += 2 * U * g_x.abs() + half * (g_x.abs() + g_x_err)
        g_x[~inside], g_x_err[~inside] = g_x0.double()[~inside], 0.0
        out.update(g_x=(g_x, g_x_err), g_a=(g_a, g_a_err), g_b=(g_b, g_b_err))
    return out


def logprobs(z, targets, top=0, g_logp=None, g_entropy=None):
    """{name: (value, largest error)} of rows of finite logits and -inf, one finite one at least in each row.

    An exponential e^d with d = z - m: d is rounded once, the product by log2(e) twice (log2(e) itself is), the power is good to two
    units: (3 |d| + 2) u.  A sum of n of them: n / 256 additions a lane and twenty beside."""
    t = z.dtype
    z = z.double()
    rows, V = z.shape
    m = z.max(1, keepdim=True).values
    d = z - m
    e = torch.exp(d)
    dz = torch.where(e > 0, d, 0.0)
    S = e.sum(1, keepdim=True)
    logS = torch.log(S)
    adds = V / 256 + 24
    s_rel = ((e * (3 * dz.abs() + 2)).sum(1, keepdim=True) / S + adds) * U       # of S, and absolute of log S
    log_err = s_rel + 3 * U * logS.abs() + 2 * U
    W = (e * dz).sum(1, keepdim=True) / S
    w_err = ((e * dz.abs() * (3 * dz.abs() + 4)).sum(1, keepdim=True) / S + adds * W.abs()) * U + W.abs() * (s_rel + 2 * U)
    H = logS - W
    h_err = log_err + w_err + U * H.abs()
    lp = d - logS
    lp_err = U * dz.abs() + log_err + U * lp.abs()
    scored = (targets >= 0) & (targets < V)
    at = targets.clamp(0, V - 1)[:, None]
    out = {"logp": (torch.where(scored, lp.gather(1, at)[:, 0], 0.0), torch.where(scored, lp_err.gather(1, at)[:, 0], 0.0)),
           "entropy": (H[:, 0], h_err[:, 0]), "stats": (torch.cat([m, logS], 1), torch.cat([0 * m, log_err], 1))}
    if top:
        ids = torch.argsort(-z, dim=1, stable=True)[:, :top]
        out["top_ids"] = ids
        out["top_logp"] = (lp.gather(1, ids), torch.where(lp.gather(1, ids) > -math.inf, lp_err.gather(1, ids), 0.0))
    if g_logp is not None or g_entropy is not None:
        gl = torch.zeros(rows, 1, dtype=torch.float64) if g_logp is None else torch.where(scored, g_logp.double(), 0.0)[:, None]
        gh = torch.zeros(rows, 1, dtype=torch.float64) if g_entropy is None else g_entropy.double()[:, None]
        p = torch.exp(lp)
        lpz = torch.where(p > 0, lp, 0.0)
        q = -gl - gh * (lpz + H)
        g = p * q
        p_rel = (3 * lpz.abs() + 2) * U + lp_err.nan_to_num(0.0, 0.0, 0.0)
        q_err = gh.abs() * (lp_err.nan_to_num(0.0, 0.0, 0.0) + h_err + 3 * U * (lpz.abs() + H.abs())) + 2 * U * gl.abs()
        err = p * (q.abs() * (p_rel + U) + q_err)
        g.scatter_add_(1, at, gl)
        err += U * g.abs() + 2.0 ** -126 * (gl.abs() + gh.abs())
        out["g_logits"] = (g, err + HALF[t] * (g.abs() + err))
    return out


# ---- the optimiser: fp32 as it is defined, operation by operation -----------------------------------------------------

def held_m(t, nearest):
    """Codes and exponents of fp32 t (a multiple of 32 long, finite)."""
    g = t.reshape(-1, 32)
    e = np.clip((np.abs(g).max(1).astype(np.float32).view(np.uint32) + 0x10000) >> 23, 8, 254).astype(np.int64)
    v = g * ((260 - e) << 23).astype(np.uint32).view(np.float32)[:, None]
    if nearest:
        c = np.rint(v)
    else:
        low = np.floor(v)
        c = low + ((v - low) > (v.view(np.uint32) & 0x7FF).astype(np.float32) / np.float32(2048))
    return np.clip(c, -127, 127).astype(np.int8).reshape(-1), e.astype(np.uint8)


def held_v(t, nearest):
    b = t.reshape(-1, 32).view(np.uint32).astype(np.int64)
    if nearest:
        k = (b + 0x7FFFF + ((b >> 20) & 1)) >> 20
    else:
        k = (b >> 20) + ((b & 0xFFFFF) > ((b & 0x7FF) << 9))
    e = np.clip((k >> 3).max(1), 32, 254)
    c = np.where(b == 0, 0, np.clip(k - ((e - 31) * 8)[:, None], 1, 255))
    return c.astype(np.uint8).reshape(-1), e.astype(np.uint8)


def read_m(codes, e):
    return (codes.reshape(-1, 32).astype(np.float32) * ((e.astype(np.uint32) - 6) << 23).view(np.float32)[:, None]).reshape(-1)


def read_v(codes, e):
    c = codes.reshape(-1, 32).astype(np.int64)
    bits = ((c + ((e.astype(np.int64) - 31) * 8)[:, None]) << 20).astype(np.uint32)
    return np.where(c > 0, bits.view(np.float32), np.float32(0)).reshape(-1)


def pack_state(codes, e):
    """Codes and exponents of whole blocks of 1024 as bytes."""
    return np.concatenate([codes.view(np.uint8).reshape(-1, 1024), e.reshape(-1, 32)], 1).reshape(-1)


def unpack_state(buf, moment):
    b = buf.reshape(-1, 1056)
    codes = np.ascontiguousarray(b[:, :1024]).reshape(-1)
    return (codes.view(np.int8) if moment == "m" else codes), np.ascontiguousarray(b[:, 1024:]).reshape(-1)


def moments(m, v, g, beta1, beta2, factor=1.0):
    f = np.float32
    g = g * f(factor)
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + (g * f(1 - beta2)) * g


def weights(p, m, v, lr, decay, c1, c2, eps):
    """New weights in 64 bits from fp32 moments, and the largest error of fp32: four units in the step, two roundings of the sum."""
    p, m, v = (t.astype(np.float64) for t in (p, m, v))
    move = lr * (m / c1) / (np.sqrt(v / c2) + eps)
    out = p - (lr * decay * p + move)
    return out, U * (10 * np.abs(move) + 4 * np.abs(lr * decay * p) + 2 * np.abs(p))
