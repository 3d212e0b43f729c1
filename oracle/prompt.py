"""Prompts into the paged cache, causal attention over packed prompts, and a
cache in 8 bits (oracle, float64).

Test infrastructure: see the package docstring.  None of this is in the paper:
these are the operators that fill the cache which its decode step reads, so
nothing here is pinned to it ("parity unpinned").
"""
from __future__ import annotations

import math

import numpy as np

BS = 16
BAD_TABLE, BAD_CTXLEN, CACHE_FULL = 1, 2, 4
TOP, MIN_EXP = 448.0, -64


def plan(n_new, ctx_lens, tables, free_ids, free_range, max_tokens: int, num_pool_blocks: int):
    """Places of a batch's new tokens, request by request (see ent_prompt_plan).

    Returns (tables, starts, slots, new_lens, free_range, flags); the inputs
    are left alone."""
    tables = np.array(tables)
    B, maxb = tables.shape
    head, end = int(free_range[0]), int(free_range[1])
    flags = 0
    ok = 0 <= head <= end <= len(free_ids)
    if not ok:
        flags |= BAD_TABLE
    starts, slots, lens = [0], [], []
    stop = not ok                     # a bad range serves nobody, also who needs no block
    at = head
    for b in range(B):
        n, ctx = int(n_new[b]), int(ctx_lens[b])
        if n < 0 or ctx < 0 or ctx > maxb * BS:
            flags |= BAD_CTXLEN
            n = 0
        elif ctx + n > maxb * BS:
            flags |= CACHE_FULL
            n = 0
        have = -(-max(ctx, 0) // BS)
        need = -(-(ctx + n) // BS) - have if n else 0
        if n and (stop or len(slots) + n > max_tokens or at + need > end):
            stop = True
            flags |= CACHE_FULL
            n = need = 0
        for j in range(have, have + need):
            p = int(free_ids[at])
            at += 1
            if not 0 <= p < num_pool_blocks:
                flags |= BAD_TABLE
                p = -1
            tables[b, j] = p
        for pos in range(ctx, ctx + n):
            p = int(tables[b, pos // BS])
            if not 0 <= p < num_pool_blocks:
                flags |= BAD_TABLE
                slots.append(-1)
            else:
                slots.append(p * BS + pos % BS)
        starts.append(len(slots))
        lens.append(ctx + n)
    slots += [-1] * (max_tokens - len(slots))
    return (tables, np.array(starts, np.int32), np.array(slots, np.int64), np.array(lens, np.int32),
            np.array([at if ok else free_range[0], free_range[1]], np.int32), flags)


def attention(q, k, v, starts, scale: float):
    """Causal attention over packed requests: q [T, H_q, d]; k, v [T, H_kv, d].

    Returns (out [T, H_q, d], lse [T, H_q], mass [T, H_q, d], span [T, H_q]): mass is
    the attention over |v|, span the largest scale sum_d |q_d k_d| of a row; both
    serve error bounds.  Rows from starts[-1] on are NaN."""
    T, Hq, d = q.shape
    G = Hq // k.shape[1]
    out = np.full((T, Hq, d), np.nan)
    lse, mass, span = np.full((T, Hq), np.nan), np.full((T, Hq, d), np.nan), np.full((T, Hq), np.nan)
    for a, e in zip(starts[:-1], starts[1:]):
        a, e = int(a), int(e)
        seen = np.tril(np.ones((e - a, e - a), bool))
        for h in range(Hq if e > a else 0):
            x = q[a:e, h]
            s = np.where(seen, scale * (x @ k[a:e, h // G].T), -np.inf)
            m = s.max(1, keepdims=True)
            w = np.exp(s - m)
            l = w.sum(1, keepdims=True)
            out[a:e, h] = (w @ v[a:e, h // G]) / l
            mass[a:e, h] = (w @ np.abs(v[a:e, h // G])) / l
            lse[a:e, h] = (m + np.log(l))[:, 0]
            span[a:e, h] = np.where(seen, abs(scale) * (np.abs(x) @ np.abs(k[a:e, h // G]).T), 0).max(1)
    return out, lse, mass, span


def store(k_pool, v_pool, ksum, slots, k, v):
    """Packed rows k, v [T, H_kv, d] at their slots (-1: skipped), in place, and the
    mean key of every block written, over its slots up to the last one written."""
    last = {}
    for t, s in enumerate(slots):
        if s < 0:
            continue
        p, i = int(s) // BS, int(s) % BS
        k_pool[p, :, i] = k[t]
        v_pool[p, :, :, i] = v[t]
        last[p] = max(last.get(p, 0), i + 1)
    for p, n in last.items():
        ksum[p] = k_pool[p, :, :n].mean(1)


def e4m3_values() -> np.ndarray:
    """Value of each of the 256 codes (4 exponent bits of bias 7, 3 of mantissa, no
    infinities; 0x7f and 0xff are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    x = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    x = np.where((c & 0x7f) == 0x7f, np.nan, x)
    return np.where(c & 0x80, -x, x)


def e4m3_round(x):
    """Nearest e4m3 value, ties to even, saturating; NaN stays NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0.0, x)), TOP)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.where(np.isnan(x), np.nan, np.copysign(np.rint(a / step) * step, x))


def scale8(x) -> float:
    """The smallest 2^k, k >= MIN_EXP, with 448 2^k >= every finite |x|."""
    a = np.abs(x[np.isfinite(x)])
    top = float(a.max()) if a.size else 0.0
    k = MIN_EXP
    while TOP * 2.0 ** k < top:
        k += 1
    return 2.0 ** k


def _tile8(codes, scale, rows, first):
    """One tile's codes [16, d] and scale after rows [n, d] at slots first ..."""
    need = scale8(rows)
    s = max(need, scale) if first else need
    codes = codes.copy()
    if first and s > scale:
        # In float32, as for every scale: exact for powers of two.
        f = np.float32(scale) / np.float32(s)
        codes[:first] = e4m3_round(codes[:first].astype(np.float32) * f)
    inv = np.float32(1.0) / np.float32(s)
    codes[first:first + len(rows)] = e4m3_round(rows.astype(np.float32) * inv)
    return codes, s


def store8(k_codes, v_codes, k_scale, v_scale, ksum, slots, k, v):
    """store into an 8-bit cache, in place: k_codes [P, H, 16, d] and v_codes
    [P, H, d, 16] hold code values, k_scale and v_scale [P, H] their tiles' scales."""
    t = 0
    while t < len(slots):
        s = int(slots[t])
        n = 1
        if s >= 0:
            while t + n < len(slots) and slots[t + n] == s + n and (s + n) % BS:
                n += 1
            p, first = s // BS, s % BS
            for g in range(k.shape[1]):
                c, k_scale[p, g] = _tile8(k_codes[p, g], float(k_scale[p, g]), k[t:t + n, g], first)
                k_codes[p, g] = c
                ksum[p, g] = c[:first + n].mean(0) * k_scale[p, g]
                c, v_scale[p, g] = _tile8(v_codes[p, g].T, float(v_scale[p, g]), v[t:t + n, g], first)
                v_codes[p, g] = c.T
        t += n
