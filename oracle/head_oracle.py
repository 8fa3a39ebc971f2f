"""The losses of a language model's head in numpy fp64, row by row of their definitions.

Cross entropy: loss = log sum_v exp(z_v) - z_y, z = W h.  Distillation: with the teacher's entries (index_j, s_j),
q = softmax(s / tau), p = softmax(z / tau): loss = tau^2 sum_j q_j (log q_j - log p_index(j)).  Entries that are none (a negative
index, a teacher's logit of -inf) are left out; a token without entries, or without target, has loss 0 and no gradient; an index of
vocab or more makes the loss nan and gives no gradient.
"""
from __future__ import annotations

import numpy as np


def softmax_row(z):
    """(probabilities, log of the sum of exponentials) of one row."""
    top = np.max(z)
    e = np.exp(z - top)
    return e / e.sum(), top + np.log(e.sum())


def head_loss(hidden, weight, targets=None, index=None, teacher=None, tau=1.0, scale=None):
    """dict(loss, lse, d_hidden, d_weight, d_logits); the gradients are those of sum(scale * loss)."""
    tokens, vocab = hidden.shape[0], weight.shape[0]
    scale = np.ones(tokens) if scale is None else np.asarray(scale, dtype=np.float64)
    loss, lse, dz = np.zeros(tokens), np.zeros(tokens), np.zeros((tokens, vocab))
    for t in range(tokens):
        with np.errstate(all="ignore"):
            z = weight @ hidden[t] / tau
            p, lse[t] = softmax_row(z)
        if targets is not None:
            entries = [(int(targets[t]), 0.0)] if targets[t] >= 0 else []
        else:
            entries = [(int(v), s / tau) for v, s in zip(index[t], teacher[t]) if v >= 0 and not s == -np.inf]
            if any(v >= vocab for v in index[t]):
                entries = [(vocab, 0.0)]
        if any(v >= vocab for v, _ in entries):
            loss[t] = np.nan
            continue
        if not entries:
            continue
        q, norm = softmax_row(np.array([s for _, s in entries]))
        want = np.zeros(vocab)
        for (v, s), w in zip(entries, q):
            loss[t] += tau * tau * w * (s - norm - z[v] + lse[t])
            want[v] += w
        if scale[t] != 0.0:
            dz[t] = scale[t] * tau * (p - want)
    live = np.any(dz != 0.0, axis=1)
    d_weight = np.zeros_like(weight)
    d_weight += dz[live].T @ hidden[live]
    return {"loss": loss, "lse": lse, "d_hidden": dz @ weight, "d_weight": d_weight, "d_logits": dz}
