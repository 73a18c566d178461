"""fp64 oracle of the token log probabilities, their entropy, alternatives and
gradient, from the definitions: one row at a time, numpy only."""
from __future__ import annotations

import math

import numpy as np


def row(z, x):
    """(logprob of column x, entropy, log-sum-exp) of logits z [V]; columns of -infinity have probability 0."""
    z = np.asarray(z, dtype=np.float64)
    m = float(z.max())
    if m == -math.inf:
        return math.nan, math.nan, -math.inf
    lse = m + math.log(float(np.exp(z - m).sum()))
    live = z[z > -math.inf]
    p = np.exp(live - lse)
    return float(z[x]) - lse, -float((p * (live - lse)).sum()), lse


def alternatives(z, k):
    """Columns of the k largest logits, the lowest column of equal ones first; NaN is none (-1)."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    order = np.argsort(-z, kind="stable")          # NaN last
    order = order[~np.isnan(z[order])][:k]
    return np.concatenate([order, np.full(k - len(order), -1)]).astype(np.int64)


def row_grad(z, x, lse, entropy, dlogprob, dentropy):
    """Gradient of dlogprob * logprob + dentropy * entropy to z, with the forward's lse and entropy."""
    z = np.asarray(z, dtype=np.float64)
    live = z > -math.inf
    lp = np.where(live, z, 0.0) - lse
    p = np.where(live, np.exp(lp), 0.0)
    g = -dlogprob * p - dentropy * p * (lp + entropy)
    g[x] += dlogprob
    return g
