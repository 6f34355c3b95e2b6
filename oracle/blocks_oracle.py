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
