"""float64 oracle of the router, the mix, and the expert and adapter layers.

Plain numpy, one group at a time, written from the formulas.  Sums of products come with the
sum of the products' magnitudes, the scale of a rounded sum's error.
"""
from __future__ import annotations

import numpy as np


def logistic(x):
    return 1.0 / (1.0 + np.exp(-x))


# ------------------------------------------------------------------ router
def route(z, k, gates):
    """(expert, gate, offsets, source, place) of logits z [n, E]; gates "chosen" or "all"."""
    n, E = z.shape
    expert = np.full((n, k), -1, dtype=np.int32)
    gate = np.zeros((n, k))
    for t in range(n):
        open_ = [e for e in range(E) if z[t, e] > -np.inf]   # not NaN, not closed
        best = sorted(open_, key=lambda e: (-z[t, e], e))[:k]
        if not best:
            continue
        expert[t, :len(best)] = best
        over = z[t, best] if gates == "chosen" else z[t]
        peak = z[t, best[0]]
        with np.errstate(invalid="ignore"):
            total = np.exp(over - peak).sum()
            gate[t, :len(best)] = np.exp(z[t, best] - peak) / total
        if np.isnan(z[t]).any():
            gate[t, :len(best)] = np.nan
    rows = [(e, t, j) for t in range(n) for j, e in enumerate(expert[t]) if e >= 0]
    rows.sort(key=lambda r: (r[0], r[1]))
    offsets = np.zeros(E + 1, dtype=np.int32)
    source = np.full(n * k, -1, dtype=np.int32)
    place = np.full((n, k), -1, dtype=np.int32)
    for r, (e, t, j) in enumerate(rows):
        offsets[e + 1:] += 1
        source[r] = t
        place[t, j] = r
    return expert, gate, offsets, source, place


def route_backward(z, expert, gate, dgate, gates):
    n, E = z.shape
    out = np.zeros((n, E))
    for t in range(n):
        s = [j for j, e in enumerate(expert[t]) if e >= 0]
        if not s:
            continue
        pull = sum(gate[t, j] * dgate[t, j] for j in s)
        if gates == "all":
            p = np.exp(z[t] - z[t].max())
            out[t] = -p / p.sum() * pull
        for j in s:
            out[t, expert[t, j]] += gate[t, j] * (dgate[t, j] - (pull if gates == "chosen" else 0.0))
    return out


# ------------------------------------------------------------------ mix
def scores_of(z, kind):
    """Softmax or sigmoid scores of the logits; 0 for a logit of -infinity or NaN (among those that are none)."""
    closed = ~(z > -np.inf)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        if kind == "sigmoid":
            p = 1.0 / (1.0 + np.exp(-z))
        else:
            peak = np.max(np.where(closed, -np.inf, z), axis=1, keepdims=True)
            up = np.where(z == peak, 1.0, np.exp(z - peak))   # (infinite logits too)
            up[closed] = 0.0
            p = up / up.sum(1, keepdims=True)
    return np.where(closed, 0.0, p)


def route_scored(z, bias, k, kind, n_groups=1, open_groups=1, group_top=1, renormalise=False, scale=1.0):
    """(expert, gate, offsets, source, place) of logits z [n, E] by scores and a bias [E] (None: 0)."""
    n, E = z.shape
    b = np.zeros(E) if bias is None else bias
    p = scores_of(z, kind)
    c = np.where((z > -np.inf) & (b > -np.inf), p + b, -np.inf)
    if n_groups > 1:
        by = np.sort(c.reshape(n, n_groups, -1), axis=2)[:, :, ::-1]
        worth = by[:, :, 0].copy()
        if group_top == 2 and by.shape[2] > 1:
            two = by[:, :, 1] > -np.inf
            worth[two] += by[:, :, 1][two]
        best = np.argsort(-worth, axis=1, kind="stable")[:, :open_groups]
        stays = np.zeros((n, n_groups), dtype=bool)
        np.put_along_axis(stays, best, True, axis=1)
        c = np.where(np.repeat(stays, E // n_groups, axis=1), c, -np.inf)
    expert = np.argsort(-c, axis=1, kind="stable")[:, :k].astype(np.int32)
    chosen = np.take_along_axis(c, expert, 1) > -np.inf
    gate = np.where(chosen, scale * _shares(z, p, expert, chosen, kind, renormalise), 0.0)
    gate[np.isnan(z).any(1, keepdims=True) & chosen] = np.nan
    expert[~chosen] = -1
    flat = expert.ravel().astype(np.int64)
    rows = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))]).astype(np.int32)
    source, place = np.full(n * k, -1, dtype=np.int32), np.full(n * k, -1, dtype=np.int32)
    rows = rows[:offsets[E]]
    source[:len(rows)] = rows // k
    place[rows] = np.arange(len(rows))
    return expert, gate, offsets, source, place.reshape(n, k)


def _shares(z, p, expert, chosen, kind, renormalise):
    """Scores of the chosen experts, or their parts of the sum, by logarithms (which do not vanish)."""
    if not renormalise:
        return np.where(chosen, np.take_along_axis(p, np.maximum(expert, 0), 1), 0.0)
    zc = np.take_along_axis(z, np.maximum(expert, 0), 1)
    a = np.minimum(zc, 0.0) if kind == "sigmoid" else zc
    peak = np.max(np.where(chosen, a, -np.inf), axis=1, keepdims=True)
    with np.errstate(invalid="ignore"):
        w = np.where(a == peak, 1.0, np.exp(a - peak))
        if kind == "sigmoid":
            w = w / (1.0 + np.exp(-np.abs(zc)))
    w = np.where(chosen, w, 0.0)
    total = w.sum(1, keepdims=True)
    return w / np.where(total > 0, total, 1.0)


def route_scored_backward(z, expert, dgate, kind, renormalise=False, scale=1.0):
    """The gates' gradient by the logits, and the magnitudes of its terms."""
    out, mag = np.zeros(z.shape), np.zeros(z.shape)
    p, chosen = scores_of(z, kind), expert >= 0
    share = _shares(z, p, expert, chosen, kind, renormalise)
    u = np.where(chosen, scale * dgate, 0.0)
    pull, pull_mag = (share * u).sum(1, keepdims=True), (share * np.abs(u)).sum(1, keepdims=True)
    if kind == "softmax" and not renormalise:
        out, mag = -p * pull, p * pull_mag
    at = np.maximum(expert, 0)
    if renormalise or kind == "softmax":
        d, m = share * (u - pull), share * (np.abs(u) + pull_mag)
    else:
        d, m = share * u, share * np.abs(u)
    if kind == "sigmoid":
        with np.errstate(over="ignore"):
            d, m = (x / (1.0 + np.exp(np.take_along_axis(z, at, 1))) for x in (d, m))
    for j in range(expert.shape[1]):
        t = np.nonzero(chosen[:, j])[0]
        out[t, expert[t, j]], mag[t, expert[t, j]] = d[t, j], m[t, j]
    return out, mag


def mix(H, place, gate):
    y = np.zeros((place.shape[0], H.shape[1]))
    for t in range(place.shape[0]):
        for j, r in enumerate(place[t]):
            if 0 <= r < H.shape[0]:
                y[t] += gate[t, j] * H[r]
    return y


def mix_backward(D, H, place, gate, dH):
    """dgate; rows of dH that a place names are rewritten."""
    dgate = np.zeros(place.shape)
    for t in range(place.shape[0]):
        for j, r in enumerate(place[t]):
            if 0 <= r < H.shape[0]:
                dH[r] = gate[t, j] * D[t]
                dgate[t, j] = D[t] @ H[r]
    return dgate


# ------------------------------------------------------------------ experts
def _groups(offsets):
    return [(g, int(offsets[g]), int(offsets[g + 1])) for g in range(len(offsets) - 1)]


def experts_forward(W, b, X, source, offsets, n_rows):
    """Sums W_e x + b_e [n_rows, n_out] and their magnitudes (0 for rows in no group)."""
    x = X if source is None else X[np.clip(source, 0, X.shape[0] - 1)]
    y = np.zeros((n_rows, W.shape[1]))
    mag = np.zeros_like(y)
    for g, lo, hi in _groups(offsets):
        y[lo:hi] = x[lo:hi] @ W[g].T + (0 if b is None else b[g])
        mag[lo:hi] = np.abs(x[lo:hi]) @ np.abs(W[g].T) + (0 if b is None else np.abs(b[g]))
    return y, mag


def experts_backward(W, X, source, offsets, D, squash):
    """dX, G_W, G_b, each with the magnitudes of its sums."""
    x = X if source is None else X[np.clip(source, 0, X.shape[0] - 1)]
    x = x[:D.shape[0]]
    E, n_out, n_in = W.shape
    dX, mX = np.zeros((D.shape[0], n_in)), np.zeros((D.shape[0], n_in))
    GW, mW = np.zeros(W.shape), np.zeros(W.shape)
    Gb, mb = np.zeros((E, n_out)), np.zeros((E, n_out))
    for g, lo, hi in _groups(offsets):
        d = D[lo:hi]
        slope = x[lo:hi] * (1 - x[lo:hi]) if squash else np.ones((hi - lo, n_in))
        dX[lo:hi] = d @ W[g] * slope
        mX[lo:hi] = np.abs(d) @ np.abs(W[g]) * np.abs(slope)
        GW[g], mW[g] = d.T @ x[lo:hi], np.abs(d).T @ np.abs(x[lo:hi])
        Gb[g], mb[g] = d.sum(0), np.abs(d).sum(0)
    return (dX, mX), (GW, mW), (Gb, mb)


# ------------------------------------------------------------------ adapters
def adapters_forward(W, b, A, B, scale, X, offsets, adapter):
    """(sums, magnitudes) and (U, magnitudes)."""
    y = X @ W.T + (0 if b is None else b)
    my = np.abs(X) @ np.abs(W.T) + (0 if b is None else np.abs(b))
    U, mU = np.zeros((X.shape[0], A.shape[1])), np.zeros((X.shape[0], A.shape[1]))
    for (i, lo, hi), a in zip(_groups(offsets), adapter):
        if a < 0:
            continue
        c = 1.0 if scale is None else scale[a]
        U[lo:hi], mU[lo:hi] = X[lo:hi] @ A[a].T, np.abs(X[lo:hi]) @ np.abs(A[a].T)
        y[lo:hi] += c * (U[lo:hi] @ B[a])
        my[lo:hi] += np.abs(c) * (mU[lo:hi] @ np.abs(B[a]))
    return (y, my), (U, mU)


def adapters_backward(W, A, B, scale, X, U, offsets, adapter, D, squash):
    """dX, G_A, G_B, each with the magnitudes of its sums."""
    dX, mX = D @ W, np.abs(D) @ np.abs(W)
    GA, mA, GB, mB = np.zeros(A.shape), np.zeros(A.shape), np.zeros(B.shape), np.zeros(B.shape)
    for (i, lo, hi), a in zip(_groups(offsets), adapter):
        if a < 0:
            continue
        c = 1.0 if scale is None else scale[a]
        d, x, u = D[lo:hi], X[lo:hi], U[lo:hi]
        v, mv = c * d @ B[a].T, np.abs(c) * np.abs(d) @ np.abs(B[a].T)
        dX[lo:hi] += v @ A[a]
        mX[lo:hi] += mv @ np.abs(A[a])
        GA[a] += v.T @ x
        mA[a] += mv.T @ np.abs(x)
        GB[a] += c * (u.T @ d)
        mB[a] += np.abs(c) * (np.abs(u).T @ np.abs(d))
    if squash:
        dX, mX = dX * X * (1 - X), mX * np.abs(X * (1 - X))
    return (dX, mX), (GA, mA), (GB, mB)
