"""Plain 64-bit forms of the expert layer (router, grouped products, tokens to their groups and back) and of the dropout
over tokens, each with its gradient by formula, in numpy.  Inputs are the values that the kernels see; nothing is rounded
here but the router's keys, whose fp32 sum is part of their definition."""
import numpy as np


def _f64(a):
    return np.asarray(a, dtype=np.float64)


# --------------------------------------------------------------------------- router
def route(z, k, normalise, bias=None, row_weight=None):
    """(chosen, weights, slots, offsets)."""
    z = np.asarray(z, np.float64)
    rows, experts = z.shape
    with np.errstate(invalid="ignore"):
        key = z.astype(np.float32)
        if bias is not None:
            key = key + np.asarray(bias, np.float32)
    chosen, weights = np.full((rows, k), -1, np.int64), np.zeros((rows, k))
    for r in range(rows):
        if row_weight is not None and row_weight[r] == 0:
            continue
        if np.isnan(z[r]).any() or (z[r] == np.inf).any():
            weights[r] = np.nan
            continue
        there = [e for e in range(experts) if key[r, e] > -np.inf]
        best = sorted(there, key=lambda e: (-key[r, e], e))[:k]
        if not best:
            continue
        over = z[r][best] if normalise else z[r]
        if over.max() == -np.inf:  # chosen by the bias alone: cannot be, the key would be -infinity
            continue
        chosen[r, :len(best)] = best
        weights[r, :len(best)] = np.exp(z[r][best] - over.max()) / np.exp(over - over.max()).sum()
    slots, offsets = group(chosen, experts)
    return chosen, weights, slots, offsets


def group(chosen, experts):
    """(slots, offsets) of the entries, by expert, then in the order they have."""
    flat = np.asarray(chosen).reshape(-1)
    slots, offsets, at = np.full(flat.size, -1, np.int64), np.zeros(experts + 1, np.int64), 0
    for e in range(experts):
        mine = np.nonzero(flat == e)[0]
        slots[mine] = at + np.arange(mine.size)
        at += mine.size
        offsets[e + 1] = at
    return slots.reshape(np.shape(chosen)), offsets


def route_bwd(z, chosen, weights, dweights, normalise):
    """(dz, size): size holds the magnitudes of the terms whose sum is dz."""
    z, w, dw = _f64(z), _f64(weights), _f64(dweights)
    dz, size = np.zeros(z.shape), np.zeros(z.shape)
    for r in range(z.shape[0]):
        if np.isnan(w[r]).any():
            dz[r] = np.nan
            continue
        there = np.nonzero(chosen[r] >= 0)[0]
        if not there.size:
            continue
        d, big = (w[r, there] * dw[r, there]).sum(), np.abs(w[r, there] * dw[r, there]).sum()
        if not normalise:
            p = np.exp(z[r] - z[r].max())
            p /= p.sum()
            dz[r], size[r] = -p * d, p * big
        for j in there:
            e = chosen[r, j]
            dz[r, e] += w[r, j] * dw[r, j] - (w[r, j] * d if normalise else 0)
            size[r, e] += abs(w[r, j] * dw[r, j]) + (w[r, j] * big if normalise else 0)
    return dz, size


# --------------------------------------------------------------------------- grouped products
def _groups(offsets, rows):
    """(group, first row, end) of offsets that may be anything: in order and inside the rows."""
    off = np.maximum.accumulate(np.clip(np.asarray(offsets, np.int64), 0, rows))
    return [(g, off[g], off[g + 1]) for g in range(off.size - 1)]


def grouped_fwd(x, w, offsets, relu=False):
    """(y, live): rows of no group are 0 in y and False in live."""
    x, w = _f64(x), _f64(w)
    y, live = np.zeros((x.shape[0], w.shape[1])), np.zeros(x.shape[0], bool)
    for g, a, b in _groups(offsets, x.shape[0]):
        y[a:b] = x[a:b] @ w[g].T
        live[a:b] = True
    return (np.where(y < 0, 0.0, y) if relu else y), live


def grouped_dgrad(dy, w, offsets, mask=None):
    dy, w = _f64(dy), _f64(w)
    dx, live = np.zeros((dy.shape[0], w.shape[2])), np.zeros(dy.shape[0], bool)
    for g, a, b in _groups(offsets, dy.shape[0]):
        dx[a:b] = dy[a:b] @ w[g]
        live[a:b] = True
    return (dx if mask is None else np.where(_f64(mask) > 0, dx, 0.0)), live


def grouped_wgrad(x, dy, offsets):
    x, dy = _f64(x), _f64(dy)
    return np.stack([dy[a:b].T @ x[a:b] for _, a, b in _groups(offsets, x.shape[0])])


# --------------------------------------------------------------------------- tokens to groups and back
def _entries(slots, grouped_rows):
    for r in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            yield r, j, slots[r, j] if 0 <= slots[r, j] < grouped_rows else -1


def scatter(x, slots, grouped):
    """grouped with the entries' rows overwritten."""
    out = _f64(grouped).copy()
    for r, _, s in _entries(slots, out.shape[0]):
        if s >= 0:
            out[s] = x[r]
    return out


def combine(yg, slots, weights=None, res=None):
    """(out, size): size holds the magnitudes of the terms."""
    yg = _f64(yg)
    out = np.zeros((slots.shape[0], yg.shape[1])) if res is None else _f64(res).copy()
    size = np.abs(out)
    for r, j, s in _entries(slots, yg.shape[0]):
        w = 1.0 if weights is None else float(weights[r, j])
        row = yg[s] if s >= 0 else np.zeros(yg.shape[1])
        out[r] += w * row
        size[r] += np.abs(w * row)
    return out, size


def combine_bwd(dout, yg, slots, weights, grouped):
    """(dyg, dweights, size): the magnitudes of dweights' terms."""
    dout, yg = _f64(dout), _f64(yg)
    dyg, dw, size = _f64(grouped).copy(), np.zeros(slots.shape), np.zeros(slots.shape)
    for r, j, s in _entries(slots, dyg.shape[0]):
        if s >= 0:
            dyg[s] = dout[r] * (1.0 if weights is None else float(weights[r, j]))
            dw[r, j], size[r, j] = (dout[r] * yg[s]).sum(), np.abs(dout[r] * yg[s]).sum()
    return dyg, dw, size


# --------------------------------------------------------------------------- dropout
def philox4x32(counter, key, rounds=10):
    """Philox4x32 of Salmon et al. (SC 2011): counter [..., 4] and key [2], 32-bit words; [..., 4] uint32."""
    mask = np.uint64(0xFFFFFFFF)
    c = [np.asarray(counter)[..., i].astype(np.uint64) for i in range(4)]
    k = [int(key[0]), int(key[1])]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & mask]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, -1).astype(np.uint32)


def dropout_mask(rows, c, rate, seed, step, row0=0):
    """True where kept, of rows row0 .. row0 + rows - 1; rate is taken as fp32."""
    per = -(-c // 4)
    block = (np.arange(rows, dtype=np.uint64)[:, None] + np.uint64(row0)) * np.uint64(per) + np.arange(per, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    counter = np.stack([block & low, block >> np.uint64(32), np.full_like(block, step & 0xFFFFFFFF),
                        np.full_like(block, step >> 32)], -1)
    words = philox4x32(counter, (seed & 0xFFFFFFFF, seed >> 32)).reshape(rows, 4 * per)[:, :c]
    return words >= np.uint32(int(np.floor(float(np.float32(rate)) * 2.0 ** 32)))


def dropout(x, rate, seed, step, res=None):
    keep = dropout_mask(x.shape[0], x.shape[1], rate, seed, step)
    y = np.where(keep, _f64(x) / (1.0 - float(np.float32(rate))), 0.0)
    return y if res is None else y + _f64(res)
