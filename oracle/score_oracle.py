"""Log probabilities of given tokens, entropies, top alternatives and their gradients in numpy fp64, row by row of their definitions."""
from __future__ import annotations

import numpy as np

from oracle.head_oracle import softmax_row


def scores(hidden, weight, targets=None, top=0, tau=1.0, d_log_prob=None, d_entropy=None):
    """dict(log_prob, entropy, lse, top_index, top_log_prob); with d_log_prob or d_entropy also d_logits, d_hidden, d_weight of
    sum(d_log_prob * log_prob + d_entropy * entropy)."""
    tokens, vocab = hidden.shape[0], weight.shape[0]
    out = {"log_prob": np.zeros(tokens), "entropy": np.zeros(tokens), "lse": np.zeros(tokens),
           "top_index": np.zeros((tokens, top), dtype=np.int64), "top_log_prob": np.zeros((tokens, top))}
    dz = np.zeros((tokens, vocab))
    for t in range(tokens):
        with np.errstate(all="ignore"):
            z = weight @ hidden[t] / tau
            p, out["lse"][t] = softmax_row(z)
            logp = z - out["lse"][t]
            plogp = np.where(p == 0.0, 0.0, p * logp)
        out["entropy"][t] = -plogp.sum()
        y = -1 if targets is None else int(targets[t])
        if y >= vocab:
            out["log_prob"][t] = np.nan
        elif y >= 0:
            out["log_prob"][t] = logp[y]
        if top:
            best = np.lexsort((np.arange(vocab), -np.where(np.isnan(z), -np.inf, z)))[:top]
            out["top_index"][t], out["top_log_prob"][t] = best, logp[best]
        g = d_log_prob[t] if d_log_prob is not None and 0 <= y < vocab else 0.0
        h = d_entropy[t] if d_entropy is not None else 0.0
        if g != 0.0:
            dz[t] -= g * p
            dz[t, y] += g
        if h != 0.0:
            dz[t] -= h * (plogp + p * out["entropy"][t])
    live = np.any(dz != 0.0, axis=1)
    out["d_logits"] = dz
    out["d_hidden"] = dz @ weight / tau
    out["d_weight"] = dz[live].T @ hidden[live] / tau
    return out
