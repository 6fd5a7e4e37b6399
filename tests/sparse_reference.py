"""Definitions of key bounds, of the choice of pages by them and of decode attention over
listed pages, on the CPU: whole numbers and float64.

Bounds and picks are whole numbers and have to be equal.  The attention's error bound is that
of chunk_reference.attend, for the tokens of the listed pages.
"""

import numpy as np

from chunk_reference import PAGE, pages_for


def power(top):
    """Least e of [-50, 50] with top <= 127 * 2^e, -7 for 0."""
    if top == 0:
        return -7
    e = -50
    while e < 50 and top > 127 * 2.0 ** e:
        e += 1
    return e


def _no_nan(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isnan(x), np.copysign(np.inf, x), x)


def page_bounds(k, length):
    """k [tokens][heads][d] (a torch tensor on the CPU): whole numbers lo, hi [pages][heads][d] and powers
    e [pages][heads] of the pages of the first `length` tokens."""
    n, (_, heads, d) = pages_for(length), k.shape
    lo, hi, e = np.zeros((n, heads, d)), np.zeros((n, heads, d)), np.zeros((n, heads), np.int64)
    k = _no_nan(k.double().numpy())
    for p in range(n):
        part = k[p * PAGE:min(length, (p + 1) * PAGE)]
        low, high = part.min(axis=0), part.max(axis=0)
        for g in range(heads):
            e[p, g] = power(max(np.abs(low[g]).max(), np.abs(high[g]).max()))
            unit = 2.0 ** e[p, g]
            lo[p, g] = np.clip(np.floor(low[g] / unit), -127, 127)
            hi[p, g] = np.clip(np.ceil(high[g] / unit), -127, 127)
    return lo, hi, e


def values(lo, hi, e):
    """What kv_read_bounds gives: [pages][heads][2][d]."""
    return np.stack([lo, hi], axis=2) * 2.0 ** e[:, :, None, None]


def scores(q, lo, hi, e):
    """q [Hq][d]: scores [heads][pages], exact."""
    q = _no_nan(q.double().numpy())
    heads, G = lo.shape[1], q.shape[0] // lo.shape[1]
    out = np.full((heads, lo.shape[0]), -np.inf)
    for h in range(q.shape[0]):
        g, eh = h // G, power(np.abs(q[h]).max())
        n = np.clip(np.rint(q[h] / 2.0 ** eh), -127, 127)
        s = (np.maximum(n, 0) * hi[:, g] + np.minimum(n, 0) * lo[:, g]).sum(axis=1)
        out[g] = np.maximum(out[g], s * 2.0 ** (eh + e[:, g].astype(np.float64)))
    return out


def choose(score, width, first, recent):
    """Picked pages (ascending) of one list with these scores [pages]."""
    n = len(score)
    if n <= width:
        return list(range(n))
    kept = [p for p in range(n) if p < first or p >= n - recent]
    rest = sorted((p for p in range(n) if p not in set(kept)), key=lambda p: (-score[p], p))
    return sorted(kept + rest[:width - len(kept)])


def attend_pages(q, k, v, length, lists, scale, dtype):
    """q [Hq][d], k, v [tokens][heads][d], lists[g] pages of KV head g: (out, bound) [Hq][d].  Pages
    outside the session's are passed over, those listed twice count twice."""
    hq, d = q.shape
    heads = k.shape[1]
    G, n = hq // heads, pages_for(length)
    q, k, v = (t.double().numpy() for t in (q, k, v))
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    uw = 2.0 ** -8 if dtype == "bf16" else 0.0
    out, bound = np.zeros((hq, d)), np.zeros((hq, d))
    for g, pages in enumerate(lists):
        at = [t for p in pages if 0 <= p < n for t in range(p * PAGE, min(length, (p + 1) * PAGE))]
        if not at:
            continue
        kk, vv, qq = k[at, g], v[at, g], q[g * G:(g + 1) * G]
        s = qq @ kk.T
        mag = np.abs(qq) @ np.abs(kk).T
        z = s * scale
        w = np.exp(z - z.max(axis=1, keepdims=True))
        w /= w.sum(axis=1, keepdims=True)
        o, A = w @ vv, w @ np.abs(vv)
        e = abs(scale) * (d + 2) * 2.0 ** -24 * mag.max(axis=1) + \
            2.0 ** -22 * (2 + abs(scale) * np.abs(s).max(axis=1))
        out[g * G:(g + 1) * G] = o
        bound[g * G:(g + 1) * G] = 1.01 * ((2 * e[:, None] + uw + 2 * (len(at) + 64) * 2.0 ** -24) * A + u * np.abs(o))
    return out, bound
