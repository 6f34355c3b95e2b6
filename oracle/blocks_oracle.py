"""float64 oracle of what stands around the layers in a model of blocks.

Plain numpy, one row or one tensor at a time, written from the formulas.  Sums come with the sum of
their terms' magnitudes, the scale of a rounded sum's error.
"""
from __future__ import annotations

import numpy as np


# ------------------------------------------------------------------ embedding
def embed(table, ids, scale):
    """Rows of the table by id, times scale; zeros for an id that names none."""
    out = np.zeros((len(ids), table.shape[1]))
    for i, t in enumerate(ids):
        if 0 <= t < len(table):
            out[i] = scale * table[t]
    return out


def embed_backward(ids, D, scale, n_tokens):
    """The change of every row of the table, and the magnitudes of its terms."""
    G, mag = np.zeros((n_tokens, D.shape[1])), np.zeros((n_tokens, D.shape[1]))
    for i, t in enumerate(ids):
        if 0 <= t < n_tokens:
            G[t] += scale * D[i]
            mag[t] += np.abs(scale * D[i])
    return G, mag


# ------------------------------------------------------------------ residual stream
NONE, RMS, LAYER = 0, 1, 2


def normed(x, kind, eps):
    """The rows normed, without weights; mean, 1 / sqrt; and the magnitude of a normed value's terms."""
    n = len(x)
    if kind == NONE:
        return x, np.zeros((n, 1)), np.ones((n, 1)), np.abs(x)
    mean = x.mean(1, keepdims=True) if kind == LAYER else np.zeros((n, 1))
    r = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * r, mean, r, r * (np.abs(x) + (np.abs(x).mean(1, keepdims=True) if kind == LAYER else 0.0))


def gate_rows(gate, offsets, n, width):
    """The gates of each row (0 for a row of no range) and which row of gates they are."""
    if gate is None:
        return np.ones((n, width)), np.zeros(n, dtype=int)
    if offsets is None:
        return np.repeat(gate, n, 0), np.zeros(n, dtype=int)
    rows, of = np.zeros((n, width)), np.full(n, -1)
    for g in range(len(gate)):
        rows[offsets[g]:offsets[g + 1]], of[offsets[g]:offsets[g + 1]] = gate[g], g
    return rows, of


def _or(x, none):
    return none if x is None else x


def residual(X, F, wo, bo, gate, offsets, scale, norm_out, eps):
    """The stream behind a block, and the magnitude of the block's part."""
    if F is None:
        return X, np.zeros(X.shape)
    f, _, _, mag = normed(F, norm_out, eps)
    k, _ = gate_rows(gate, offsets, len(X), X.shape[1])
    return X + scale * k * (f * _or(wo, 1.0) + _or(bo, 0.0)), np.abs(scale * k) * (mag * np.abs(_or(wo, 1.0)) + np.abs(_or(bo, 0.0)))


def norm_in(Y, wi, bi, kind, eps):
    """The next block's input, and the magnitude of its terms."""
    y, _, _, mag = normed(Y, kind, eps)
    return y * _or(wi, 1.0) + _or(bi, 0.0), mag * np.abs(_or(wi, 1.0)) + np.abs(_or(bi, 0.0))


def _through(d, mag_d, x, kind, eps):
    """The gradient of a norm's input by that of its normed value, and the magnitude of its terms."""
    if kind == NONE:
        return d, mag_d
    h, _, r, mag = normed(x, kind, eps)
    back = r * (d - h * (d * h).mean(1, keepdims=True) - (d.mean(1, keepdims=True) if kind == LAYER else 0.0))
    size = r * (mag_d + mag * (mag_d * mag).mean(1, keepdims=True) + (mag_d.mean(1, keepdims=True) if kind == LAYER else 0.0))
    return back, size


def residual_backward(Y, F, wo, bo, gate, offsets, scale, wi, dY, dH, norm_out, norm_in_, eps):
    """A dict of name -> (gradient, magnitude): dX, dF, Gwo, Gbo, Ggate, Gwi, Gbi."""
    out = {}
    dy, my = (np.zeros(Y.shape), np.zeros(Y.shape)) if dY is None else (dY.copy(), np.abs(dY))
    if dH is not None:
        y, _, _, mag = normed(Y, norm_in_, eps)
        d, m = _through(dH * _or(wi, 1.0), np.abs(dH * _or(wi, 1.0)), Y, norm_in_, eps)
        dy, my = dy + d, my + m
        out["Gwi"] = (dH * y).sum(0), (np.abs(dH) * mag).sum(0)
        out["Gbi"] = dH.sum(0), np.abs(dH).sum(0)
    out["dX"] = dy, my
    if F is not None:
        f, _, _, mag = normed(F, norm_out, eps)
        k, of = gate_rows(gate, offsets, len(Y), Y.shape[1])
        du, mu = scale * k * dy, np.abs(scale * k) * my
        out["Gwo"] = (du * f).sum(0), (mu * mag).sum(0)
        out["Gbo"] = du.sum(0), mu.sum(0)
        out["dF"] = _through(du * _or(wo, 1.0), mu * np.abs(_or(wo, 1.0)), F, norm_out, eps)
        if gate is not None:
            u, um = f * _or(wo, 1.0) + _or(bo, 0.0), mag * np.abs(_or(wo, 1.0)) + np.abs(_or(bo, 0.0))
            G, M = np.zeros(gate.shape), np.zeros(gate.shape)
            for t in range(len(Y)):
                if of[t] >= 0:
                    G[of[t]] += scale * dy[t] * u[t]
                    M[of[t]] += np.abs(scale) * my[t] * um[t]
            out["Ggate"] = G, M
    return out


# ------------------------------------------------------------------ clipping
def clip(tensors, max_norm):
    """(norm, the tensors times max_norm / norm where the norm is above max_norm)."""
    norm = np.sqrt(sum((x * x).sum() for x in tensors))
    return norm, [x * (max_norm / norm) for x in tensors] if norm > max_norm else tensors
