"""Log probabilities, entropy and the likeliest tokens of logit rows (oracle, float64).

Test infrastructure: see the package docstring.  The softmax is the paper's tempered one
(Section 2.1); what is returned of it is not in the paper ("parity unpinned").
"""
from __future__ import annotations

import numpy as np


def token_logprobs(z, token, T: float, n_top: int):
    """(ln p(token), entropy, ids, ln p of ids) of one row at temperature T; everything
    NaN and -1 where the row has no distribution, ln p(token) NaN past the vocabulary."""
    z = np.asarray(z, np.float64)
    ok = not np.isnan(z).any() and np.isfinite(z.max())
    if not ok:
        return np.nan, np.nan, np.full(n_top, -1), np.full(n_top, np.nan)
    t = z / T
    d = t - t.max()
    e = np.exp(d)
    lse = np.log(e.sum())
    p = e / e.sum()
    lp = d - lse
    h = -(p[p > 0] * lp[p > 0]).sum()
    ids = np.argsort(-z, kind="stable")[:n_top]
    return (lp[token] if token < len(z) else np.nan), h, ids, lp[ids]
