"""The gated recurrence in 64 bits, step by step, with bounds on what fp32 arithmetic may be off."""
import numpy as np

U = 2.0 ** -24


def sigmoid(z):
    with np.errstate(over="ignore"):
        e = np.exp(-np.abs(z))
    small = e / (1 + e)
    return np.where(z >= 0, 1 - small, small), np.where(z >= 0, small, 1 - small)


def shares(z, form):
    if form == "gate":
        return sigmoid(z)
    return z, np.ones_like(z)


def steps(a, batch):
    """[H, T * batch] as [T, H, batch]."""
    H, n = a.shape
    return np.ascontiguousarray(a.reshape(H, n // batch, batch).transpose(1, 0, 2))


def columns(a):
    return np.ascontiguousarray(a.transpose(1, 0, 2).reshape(a.shape[1], -1))


def forward(z, x, h0, resets, batch, form):
    """(h, last, bound of h's error before it is rounded to its type).

    A gate is off by at most 8 units (the exponential by 2, the sum, the reciprocal and the
    product by one each, with room), b by 10, and a step adds 2 roundings of at most the sum of
    magnitudes m: 12 units of m a step, carried on by f.  Joining maps adds two roundings a level:
    6 levels in a wave, 4 waves, at most 64 slabs, each slab's tiles among them, all of m."""
    f, u = shares(steps(z, batch), form)
    x = steps(x, batch)
    r = np.zeros((len(f), 1, batch), bool) if resets is None else resets.reshape(len(f), 1, batch) != 0
    h, m, e = h0.astype(np.float64), np.abs(h0).astype(np.float64), np.zeros_like(h0, dtype=np.float64)
    out, bound = np.empty_like(x), np.empty_like(x)
    for t in range(len(f)):
        h, m, e = (np.where(r[t], 0.0, v) for v in (h, m, e))
        h = f[t] * h + u[t] * x[t]
        m = np.abs(f[t]) * m + np.abs(u[t] * x[t])
        e = np.abs(f[t]) * e + 12 * U * m
        out[t], bound[t] = h, e + 2 * (6 + 4 + 64 + 64) * U * m
    return columns(out), h, columns(bound), bound[-1]


def backward(dh, z, x, h, h0, dh_last, resets, batch, form):
    """(dgate, dx, dh0, and each one's bound), as above."""
    f, u = shares(steps(z, batch), form)
    dh, x, h = (steps(a, batch) for a in (dh, x, h))
    r = np.zeros((len(f), 1, batch), bool) if resets is None else resets.reshape(len(f), 1, batch) != 0
    g, m = dh_last.astype(np.float64), np.abs(dh_last).astype(np.float64)
    e = np.zeros_like(g)
    dz, dx, bz, bx = (np.empty_like(x) for _ in range(4))
    for t in range(len(f) - 1, -1, -1):
        g, m = g + dh[t], m + np.abs(dh[t])
        e = e + 2 * U * m
        off = e + 2 * (6 + 4 + 64 + 64) * U * m
        past = np.where(r[t], 0.0, h[t - 1] if t else h0)
        if form == "gate":
            k = f[t] * u[t]
            dz[t], dx[t] = (past - x[t]) * g * k, g * u[t]
            bz[t] = k * (np.abs(past - x[t]) * (off + 24 * U * m) + U * (np.abs(past) + np.abs(x[t])) * m)
            bx[t] = u[t] * (off + 12 * U * m)
        else:
            dz[t], dx[t] = past * g, g
            bz[t], bx[t] = np.abs(past) * (off + 2 * U * m), off
        g, m, e = g * f[t], np.abs(f[t]) * m, np.abs(f[t]) * (e + 10 * U * m)
        g, m, e = (np.where(r[t], 0.0, v) for v in (g, m, e))
    return columns(dz), columns(dx), g, columns(bz), columns(bx), e + 2 * (6 + 4 + 64 + 64) * U * m
