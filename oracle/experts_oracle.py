"""A mixture's tokens to their experts and back, in plain Python loops and numpy fp64."""
from __future__ import annotations

import numpy as np


def sort_pairs(expert, experts):
    """(position [tokens, top], source [tokens * top], offsets [experts + 1]) of the stable sort by expert; -1 where there is none."""
    tokens, top = expert.shape
    position, source, offsets = -np.ones((tokens, top), np.int64), -np.ones(tokens * top, np.int64), [0]
    row = 0
    for e in range(experts):
        for t in range(tokens):
            for j in range(top):
                if expert[t, j] == e:
                    position[t, j], source[row] = row, t * top + j
                    row += 1
        offsets.append(row)
    return position, source, np.array(offsets, np.int64)


def dispatch(x, position):
    rows = np.zeros((position.size, x.shape[1]))
    for t, j in np.argwhere(position >= 0):
        rows[position[t, j]] = x[t]
    return rows


def combine(rows, weights, position):
    out = np.zeros((position.shape[0], rows.shape[1]))
    for t, j in np.argwhere(position >= 0):
        out[t] += (1.0 if weights is None else weights[t, j]) * rows[position[t, j]]
    return out


def combine_backward(d_out, rows, weights, position):
    d_rows, d_weights = np.zeros_like(rows), np.zeros(position.shape)
    for t, j in np.argwhere(position >= 0):
        d_rows[position[t, j]] = weights[t, j] * d_out[t]
        d_weights[t, j] = d_out[t] @ rows[position[t, j]]
    return d_rows, d_weights
