"""fp64 oracle of the latent-sequence operators: each definition written out
in NumPy, sharing nothing with the HIP path."""

import numpy as np


def rms_norm(u, w, eps):
    """(y, rstd) of rows u."""
    u = np.asarray(u, np.float64)
    rstd = 1.0 / np.sqrt((u * u).mean(axis=1) + eps)
    return u * rstd[:, None] * np.asarray(w, np.float64), rstd


def rms_norm_adj(g_y, u, w, eps, g_sum=None):
    """(g_u, g_w) of rms_norm, g_sum added to g_u."""
    g_y, u, w = (np.asarray(a, np.float64) for a in (g_y, u, w))
    _, rstd = rms_norm(u, w, eps)
    # d y_c / d u_k = w_c (rstd [c = k] - rstd^3 u_c u_k / n)
    dot = (g_y * w * u).sum(axis=1)
    g = g_y * w * rstd[:, None] - u * (dot * rstd ** 3 / u.shape[1])[:, None]
    g_w = (g_y * u * rstd[:, None]).sum(axis=0)
    return (g if g_sum is None else g + np.asarray(g_sum, np.float64)), g_w


def e4m3(v):
    """Values rounded to the nearest (ties to even) of 4 exponent and 3
    fraction bits, largest 448, smallest step 2^-9."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(np.where(np.isfinite(v), v, 0.0))
    step = np.exp2(np.maximum(e - 1, -6) - 3.0)
    r = np.round(v / step) * step
    return np.where(np.isfinite(v), r, np.nan)


def quantise(x):
    """(codes' values with the columns filled up to a multiple of 128, scale
    exponents) of rows x."""
    x = np.asarray(x, np.float64)
    r, k = x.shape
    kp = -(-k // 128) * 128
    b = np.zeros((r, kp))
    b[:, :k] = x
    b = b.reshape(r, kp // 128, 128)
    top = np.where(np.isfinite(b), np.abs(b), 0.0).max(axis=2)
    e = np.zeros(top.shape, np.int64)
    for i in np.ndindex(top.shape):
        if top[i] > 0:
            n = -126
            while top[i] > 448 * 2.0 ** n:
                n += 1
            e[i] = n
    return e4m3(b / np.exp2(e)[..., None]).reshape(r, kp), e


def values(q, e):
    """What codes (r, kp) and scale exponents (r, kp / 128) stand for."""
    return np.asarray(q, np.float64) * np.repeat(np.exp2(np.asarray(e, np.float64)), 128, axis=1)


def product(a, b, bias=None):
    r = np.asarray(a, np.float64) @ np.asarray(b, np.float64).T
    return r if bias is None else r + np.asarray(bias, np.float64)


def logistic(v):
    v = np.asarray(v, np.float64)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def recurrence(z, v, o=None, h0=None, lengths=None):
    """(y, every state (B, T + 1, F) with the first before step 0)."""
    z, v = np.asarray(z, np.float64), np.asarray(v, np.float64)
    B, T, F = z.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    h = np.zeros((B, T + 1, F))
    if h0 is not None:
        h[:, 0] = h0
    y = np.zeros((B, T, F))
    for b in range(B):
        for t in range(T):
            if t >= n[b]:
                h[b, t + 1] = h[b, t]
                continue
            s = logistic(z[b, t])
            h[b, t + 1] = s * h[b, t] + logistic(-z[b, t]) * v[b, t]
            y[b, t] = h[b, t + 1]
            if o is not None:
                ot = np.asarray(o[b, t], np.float64)
                y[b, t] = h[b, t + 1] * ot * logistic(ot)
    return y, h


def recurrence_adj(z, v, g_y, h, o=None, g_h=None, lengths=None):
    """(g_z, g_v, g_o, g_h0) from the states h of recurrence."""
    z, v, g_y = (np.asarray(a, np.float64) for a in (z, v, g_y))
    B, T, F = z.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    g_z, g_v, g_o = np.zeros((B, T, F)), np.zeros((B, T, F)), np.zeros((B, T, F))
    d = np.zeros((B, F)) if g_h is None else np.array(g_h, np.float64)
    for b in range(B):
        for t in range(int(n[b]) - 1, -1, -1):
            s, sn = logistic(z[b, t]), logistic(-z[b, t])
            g = g_y[b, t]
            if o is not None:
                ot = np.asarray(o[b, t], np.float64)
                g_o[b, t] = g * h[b, t + 1] * logistic(ot) * (1 + ot * logistic(-ot))
                g = g * ot * logistic(ot)
            d[b] += g
            g_v[b, t] = d[b] * sn
            g_z[b, t] = d[b] * (h[b, t] - v[b, t]) * s * sn
            d[b] = d[b] * s
    return g_z, g_v, g_o, d
