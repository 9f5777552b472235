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


def layer_norm(u, w, b, eps):
    """(y, mean, rstd) of rows u."""
    u = np.asarray(u, np.float64)
    mean = u.mean(axis=1)
    rstd = 1.0 / np.sqrt(((u - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (u - mean[:, None]) * rstd[:, None] * np.asarray(w, np.float64)
    return y + (0.0 if b is None else np.asarray(b, np.float64)), mean, rstd


def layer_norm_adj(g_y, u, w, eps, g_sum=None):
    """(g_u, g_w, g_b) of layer_norm, g_sum added to g_u."""
    g_y, u, w = (np.asarray(a, np.float64) for a in (g_y, u, w))
    _, mean, rstd = layer_norm(u, w, None, eps)
    n, v = u.shape[1], u - mean[:, None]
    # d y_c / d u_k = w_c (rstd ([c = k] - 1 / n) - rstd^3 v_c v_k / n)
    t = g_y * w
    g = rstd[:, None] * (t - t.sum(axis=1, keepdims=True) / n) - v * ((t * v).sum(axis=1) * rstd ** 3 / n)[:, None]
    g_w, g_b = (g_y * v * rstd[:, None]).sum(axis=0), g_y.sum(axis=0)
    return (g if g_sum is None else g + np.asarray(g_sum, np.float64)), g_w, g_b


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


def conv(x, w, bias=None, state=None, lengths=None, silu=True):
    """(y, the state after the last step)."""
    x, w = np.asarray(x, np.float64), np.asarray(w, np.float64)
    (B, T, F), K = x.shape, len(w)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    y, last = np.zeros((B, T, F)), np.zeros((B, K - 1, F))
    for i in range(B):
        z = np.zeros((K - 1 + n[i], F))
        if state is not None:
            z[:K - 1] = state[i]
        z[K - 1:] = x[i, :n[i]]
        for t in range(n[i]):
            v = (w * z[t:t + K]).sum(axis=0) + (0.0 if bias is None else np.asarray(bias, np.float64))
            y[i, t] = v * logistic(v) if silu else v
        last[i] = z[n[i]:]
    return y, last


def conv_adj(x, w, g_y, bias=None, state=None, g_last=None, lengths=None, silu=True):
    """(g_x, g_w, g_bias, g_state) of conv."""
    x, w, g_y = (np.asarray(a, np.float64) for a in (x, w, g_y))
    (B, T, F), K = x.shape, len(w)
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    g_x, g_w, g_b, g_s = np.zeros((B, T, F)), np.zeros((K, F)), np.zeros(F), np.zeros((B, K - 1, F))
    for i in range(B):
        z, gz = np.zeros((K - 1 + n[i], F)), np.zeros((K - 1 + n[i], F))
        if state is not None:
            z[:K - 1] = state[i]
        z[K - 1:] = x[i, :n[i]]
        if g_last is not None:
            gz[n[i]:] = g_last[i]
        for t in range(n[i]):
            v = (w * z[t:t + K]).sum(axis=0) + (0.0 if bias is None else np.asarray(bias, np.float64))
            p = g_y[i, t] * (logistic(v) * (1 + v * logistic(-v)) if silu else 1.0)
            gz[t:t + K] += w * p
            g_w += p * z[t:t + K]
            g_b += p
        g_s[i], g_x[i, :n[i]] = gz[:K - 1], gz[K - 1:]
    return g_x, g_w, g_b, g_s


def scan(x, delta, a, b, c, d=None, o=None, h0=None, lengths=None):
    """(y, every state (B, T + 1, N, F) with the first before step 0)."""
    x, delta, a, b, c = (np.asarray(v, np.float64) for v in (x, delta, a, b, c))
    B, T, F = x.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    h = np.zeros((B, T + 1) + a.shape)
    if h0 is not None:
        h[:, 0] = h0
    y = np.zeros((B, T, F))
    for i in range(B):
        for t in range(T):
            if t >= n[i]:
                h[i, t + 1] = h[i, t]
                continue
            D = np.logaddexp(0.0, delta[i, t])
            h[i, t + 1] = np.exp(D * a) * h[i, t] + (D * x[i, t]) * b[i, t][:, None]
            y[i, t] = (c[i, t][:, None] * h[i, t + 1]).sum(axis=0)
            if d is not None:
                y[i, t] += np.asarray(d, np.float64) * x[i, t]
            if o is not None:
                ot = np.asarray(o[i, t], np.float64)
                y[i, t] *= ot * logistic(ot)
    return y, h


def scan_adj(x, delta, a, b, c, g_y, h, d=None, o=None, g_h=None, lengths=None):
    """Gradients of x, delta, a, b, c, d, o and h0 (a dict) from the states h of scan."""
    x, delta, a, b, c, g_y = (np.asarray(v, np.float64) for v in (x, delta, a, b, c, g_y))
    B, T, F = x.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    g = {k: np.zeros(v.shape) for k, v in dict(x=x, delta=x, a=a, b=b, c=c, o=x).items()}
    g["d"] = np.zeros(F)
    q = np.zeros((B,) + a.shape) if g_h is None else np.array(g_h, np.float64)
    for i in range(B):
        for t in range(int(n[i]) - 1, -1, -1):
            D, gy = np.logaddexp(0.0, delta[i, t]), g_y[i, t]
            before, after = h[i, t], h[i, t + 1]
            if o is not None:
                ot = np.asarray(o[i, t], np.float64)
                s = (c[i, t][:, None] * after).sum(axis=0) + (0.0 if d is None else np.asarray(d, np.float64) * x[i, t])
                g["o"][i, t] = gy * s * logistic(ot) * (1 + ot * logistic(-ot))
                gy = gy * ot * logistic(ot)
            if d is not None:
                g["d"] += gy * x[i, t]
                g["x"][i, t] += gy * np.asarray(d, np.float64)
            g["c"][i, t] = (gy * after).sum(axis=1)
            q[i] += gy * c[i, t][:, None]
            g["b"][i, t] = (q[i] * D * x[i, t]).sum(axis=1)
            E = np.exp(D * a)
            qb = (q[i] * b[i, t][:, None]).sum(axis=0)
            g["x"][i, t] += D * qb
            g["delta"][i, t] = ((q[i] * E * before * a).sum(axis=0) + qb * x[i, t]) * logistic(delta[i, t])
            g["a"] += q[i] * E * before * D
            q[i] = E * q[i]
    g["h0"] = q
    return g


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
