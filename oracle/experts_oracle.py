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
