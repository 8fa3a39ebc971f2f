"""A mixture's layer in numpy fp64, pair by pair of its definition, with the magnitudes that error bounds go by."""
from __future__ import annotations

import numpy as np


def act(name, z):
    with np.errstate(over="ignore"):
        return z / (1.0 + np.exp(-z)) if name == "silu" else np.maximum(z, 0.0)


def layer(x, up, down, expert, weights=None, gate=None, activation="silu", sum_eps=0.0, h_eps=0.0):
    """(out, bound): what rounding of sums of n products (relative (4 + sqrt n) sum_eps of the sum of magnitudes) and of h (h_eps) may add
    up to in each element of out."""
    tokens, width = x.shape
    out, bound = np.zeros((tokens, width)), np.zeros((tokens, width))
    for t in range(tokens):
        for j in range(expert.shape[1]):
            e = int(expert[t, j])
            if not 0 <= e < up.shape[0]:
                continue
            w = 1.0 if weights is None else weights[t, j]
            per = (4 + np.sqrt(width)) * sum_eps
            u, u_err = x[t] @ up[e], per * (np.abs(x[t]) @ np.abs(up[e]))
            if gate is None:
                h, h_err = act(activation, u), 1.1 * u_err              # |silu'| <= 1.1
            else:
                g, g_err = x[t] @ gate[e], per * (np.abs(x[t]) @ np.abs(gate[e]))
                lead = act(activation, g)
                h, h_err = lead * u, 1.1 * g_err * (np.abs(u) + u_err) + np.abs(lead) * u_err
            h_err = h_err + np.abs(h) * (h_eps + 2.0 ** -21)             # the activation's own few roundings
            y = h @ down[e]
            y_err = h_err @ np.abs(down[e]) + (4 + np.sqrt(len(h))) * sum_eps * (np.abs(h) @ np.abs(down[e]))
            out[t] += w * y
            bound[t] += np.abs(w) * (y_err + 2.0 ** -20 * np.abs(y))
    return out, bound
