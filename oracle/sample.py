"""The next token by temperature, top-k, top-p, min-p and a given random number (oracle, test only; fp64 NumPy, one row).

Tokens in order of falling logit, equal ones by id; each filter keeps a first part of that order and the first token always; the draw is
the first kept token whose weights so far exceed u times all that are kept."""
from __future__ import annotations

import numpy as np


def kept_weights(z, temperature, top_k=0, top_p=1.0, min_p=0.0):
    """(ids in order, weights) of the kept tokens."""
    z = np.asarray(z, np.float64)
    order = np.argsort(-z, kind="stable")
    if temperature == 0:
        return order[:1], np.ones(1)
    x = (z[order] - z[order[0]]) / temperature
    w = np.exp(x)
    n = len(w)
    if 0 < top_k < n:
        n = int(top_k)
    if top_p < 1:
        total = w[:n].sum()
        before = np.concatenate([[0.0], np.cumsum(w[:n])[:-1]])
        n = max(1, int((before < top_p * total).sum()))
    if min_p > 0:
        n = max(1, min(n, int((x >= np.log(min_p)).sum())))
    return order[:n], w[:n]


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its share, distance of u from the next border in shares: how far a rounding is from another answer)."""
    ids, w = kept_weights(z, temperature, top_k, top_p, min_p)
    upto = np.cumsum(w)
    i = min(int((upto <= u * upto[-1]).sum()), len(w) - 1)
    while w[i] == 0.0:
        i -= 1
    return int(ids[i]), float(np.log(w[i] / upto[-1])), float(np.abs(upto[:-1] / upto[-1] - u).min()) if len(w) > 1 else 1.0
