"""Plain 64-bit forms of the token operators (layer norm, gated scan, distillation), each with its gradient by
formula, in numpy.  Inputs are the values that the kernels see; nothing is rounded here."""
import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


# --------------------------------------------------------------------------- layer norm
def layer_norm_fwd(x, gamma=None, beta=None, eps=1e-5, res=None):
    """(y, mean, invstd, sum): the sum is x + res, before any rounding."""
    s = _f64(x) if res is None else _f64(x) + _f64(res)
    mean = s.mean(1)
    d = s - mean[:, None]
    invstd = 1.0 / np.sqrt((d * d).mean(1) + eps)
    y = d * invstd[:, None]
    if gamma is not None:
        y = y * _f64(gamma)
    if beta is not None:
        y = y + _f64(beta)
    return y, mean, invstd, s


def layer_norm_bwd(dy, x, gamma, mean, invstd, dskip=None):
    """(dx, dgamma, dbeta)."""
    dy, x, inv = _f64(dy), _f64(x), _f64(invstd)[:, None]
    h = (x - _f64(mean)[:, None]) * inv
    g = dy if gamma is None else dy * _f64(gamma)
    dx = inv * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    if dskip is not None:
        dx = dx + _f64(dskip)
    return dx, (dy * h).sum(0), dy.sum(0)


# --------------------------------------------------------------------------- gated scan
def gates(z):
    """sigma(z) and 1 - sigma(z) (which is sigma(-z), without cancellation)."""
    z = _f64(z)
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-z)), 1.0 / (1.0 + np.exp(z))


def _lengths(n, t, lengths):
    return np.full(n, t) if lengths is None else np.clip(np.asarray(lengths), 0, t)


def gated_scan_fwd(x, z, h0=None, lengths=None, chunk=64):
    """(h, h_last, states, prev): prev[:, i] is the state before step i."""
    x = _f64(x)
    n, t, c = x.shape
    ln = _lengths(n, t, lengths)
    a, na = gates(z)
    state = np.zeros((n, c)) if h0 is None else _f64(h0).copy()
    h, prev = np.zeros((n, t, c)), np.zeros((n, t, c))
    states = np.zeros((n, -(-t // chunk), c))
    for i in range(t):
        if i % chunk == 0:
            states[:, i // chunk] = state
        prev[:, i] = state
        at = i < ln
        state = state.copy()
        state[at] = a[at, i] * state[at] + na[at, i] * x[at, i]
        h[at, i] = state[at]
    return h, state, states, prev


def gated_scan_bwd(dh, x, z, prev, dh_last=None, lengths=None):
    """(dx, dgate, dh0, whole): whole[:, i] is the whole gradient of the state after step i."""
    dh, x = _f64(dh), _f64(x)
    n, t, c = x.shape
    ln = _lengths(n, t, lengths)
    a, na = gates(z)
    q = np.zeros((n, c)) if dh_last is None else _f64(dh_last).copy()
    dx, dz, whole = np.zeros((n, t, c)), np.zeros((n, t, c)), np.zeros((n, t, c))
    for i in range(t - 1, -1, -1):
        at = i < ln
        g = dh[at, i] + q[at]
        whole[at, i] = g
        dx[at, i] = na[at, i] * g
        dz[at, i] = g * (prev[at, i] - x[at, i]) * a[at, i] * na[at, i]
        q[at] = a[at, i] * g
    return dx, dz, q, whole


# --------------------------------------------------------------------------- distillation
def distill(z, top, classes, labels=None, weight=None, temperature=1.0, alpha=1.0, scale=1.0):
    """(row_loss, loss, dz, size): size holds the magnitudes of the terms whose sum is dz."""
    z = _f64(z)
    n, v = z.shape
    top, classes = _f64(top).reshape(n, -1), np.asarray(classes).reshape(n, -1)
    w = np.full(n, 1.0 / n) if weight is None else _f64(weight)
    row, dz, size = np.zeros(n), np.zeros((n, v)), np.zeros((n, v))
    for r in range(n):
        if w[r] == 0:
            continue
        there = (classes[r] >= 0) & (classes[r] < v) & (top[r] != -np.inf)
        if alpha > 0 and there.any():
            t = top[r][there] / temperature
            p = np.exp(t - t.max())
            p /= p.sum()
            cls = classes[r][there]
            s = (z[r] - z[r].max()) / temperature
            lse = np.log(np.exp(s).sum())
            q = np.exp(s - lse)
            for pj, c in zip(p, cls):
                if pj > 0:
                    row[r] += alpha * temperature ** 2 * pj * (np.log(pj) - (s[c] - lse))
            f = w[r] * scale * alpha * temperature
            dz[r] += f * q
            size[r] += f * q
            np.add.at(dz[r], cls, -f * p)
            np.add.at(size[r], cls, f * p)
        if labels is not None and alpha < 1 and 0 <= labels[r] < v:
            s = z[r] - z[r].max()
            lse = np.log(np.exp(s).sum())
            row[r] += (1 - alpha) * (lse - s[labels[r]])
            f = w[r] * scale * (1 - alpha)
            dz[r] += f * np.exp(s - lse)
            size[r] += f * np.exp(s - lse)
            dz[r, labels[r]] -= f
            size[r, labels[r]] += f
    return row, float((w * row).sum()), dz, size
