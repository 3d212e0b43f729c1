"""Norms and rotation of queries and keys (oracle, float64).

Test infrastructure: see the package docstring.  Not in the paper ("parity unpinned"):
attention and the cache take queries and keys as this operator gives them.
"""
from __future__ import annotations

import numpy as np


def positions(T: int, starts, ctx_lens, room: int):
    """Position of each of T rows (-1: the row is left alone) and whether a length was
    out of [0, room] (see ent_qk_norm_rope).  starts None: row b is request b's."""
    pos, bad = np.full(T, -1, np.int64), False
    B = T if starts is None else len(starts) - 1
    for b in range(B):
        n = 0 if ctx_lens is None else int(ctx_lens[b])
        a, e = (b, b + 1) if starts is None else (int(starts[b]), int(starts[b + 1]))
        if n < 0 or n > room:
            bad = bad or e > a
            continue
        pos[a:e] = n + np.arange(max(0, e - a))
    return pos, bad


def norm_rope(x, pos, gain, inv_freq, eps: float, rot: int, adjacent: bool):
    """x [T, H, d] normalised (gain not None) and turned; rows of position -1 are NaN.

    Also the size of what each output is a sum of (|y_a| + |y_b|), for error bounds."""
    x = np.asarray(x, np.float64)
    y = x.copy()
    if gain is not None:
        y = x * np.asarray(gain, np.float64) / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    out, size = y.copy(), np.abs(y)
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + rot // 2)
        w = pos.astype(np.float64) * float(inv_freq[i])
        c, s = np.cos(w)[:, None], np.sin(w)[:, None]
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., b] * c + y[..., a] * s
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    out[pos < 0] = np.nan
    return out, size
