"""The calls on the paged key/value cache in float64 on the CPU, written from their definitions (include/tkphi.h): rotation by
position, means of filled blocks, attention over the tokens a query sees, selection of blocks.

Pools are float64 arrays [pages][KV heads][tokens per page][channels]; `table` holds a sequence's page ids (-1: absent)."""
from __future__ import annotations

import numpy as np


def rotate(x: np.ndarray, pos: int, inv_freq: np.ndarray, adjacent: bool) -> np.ndarray:
    """x [..., d] at position pos; the first 2 len(inv_freq) channels turn."""
    h = len(inv_freq)
    y = x.astype(np.float64).copy()
    i = 2 * np.arange(h) if adjacent else np.arange(h)
    j = i + 1 if adjacent else i + h
    z = (x[..., i] + 1j * x[..., j]) * np.exp(1j * np.longdouble(pos) * inv_freq.astype(np.longdouble))
    y[..., i], y[..., j] = z.real, z.imag
    return y


def gather(pool: np.ndarray, table, length: int):
    """Rows of the first `length` tokens [KV heads][length][d], and which of them are there."""
    page = pool.shape[2]
    t = np.arange(length)
    entry = t // page
    ids = np.array([table[e] if e < len(table) else -1 for e in entry], dtype=np.int64)
    there = (ids >= 0) & (ids < pool.shape[0])
    rows = pool[np.where(there, ids, 0), :, t % page]
    return np.swapaxes(rows, 0, 1), there


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray, seen: np.ndarray, scale: float):
    """q [d], K, V [tokens][d], seen [tokens] -> y, lse, and sum p |v| / sum p, the largest |score| terms (for error bounds)"""
    K, V = K[seen], V[seen]
    if K.shape[0] == 0:
        z = np.zeros(q.shape[0])
        return z, -np.inf, z, 0.0
    x = scale * (K @ q)
    m = x.max()
    m = m if np.isfinite(m) else 0.0
    e = np.exp(x - m)
    z = e.sum()
    if z == 0:
        zero = np.zeros(q.shape[0])
        return zero, -np.inf, zero, 0.0
    with np.errstate(invalid="ignore"):
        y = (e @ V) / z
        spread = (e @ np.abs(V)) / z
    return y, m + np.log(z), spread, float(scale * (np.abs(K) @ np.abs(q)).max())


def paged_attention(q, K, V, table, cached: int, fresh: int, scale: float, window: int = 0):
    """q [fresh][Hq][d] of one sequence -> lists of attend() results per token and head"""
    hkv = K.shape[1]
    G = q.shape[1] // hkv
    Kr, there = gather(K, table, cached + fresh)
    Vr, _ = gather(V, table, cached + fresh)
    t = np.arange(cached + fresh)
    out = []
    for i in range(fresh):
        seen = there & (t <= cached + i)
        if window:
            seen &= t > cached + i - window
        out.append([attend(q[i, g], Kr[g // G], Vr[g // G], seen, scale) for g in range(q.shape[1])])
    return out


def pick_blocks(q, M, table, block: int, page: int, pos: int, first: int, last: int, top: int):
    """q [G][d] of one token and KV head, M [pages][blocks per page][d] of that head -> sorted ids"""
    per, have = page // block, pos // block + 1
    always = [b for b in range(have) if b < first or b >= have - last]
    others = [b for b in range(have) if b not in set(always)]
    score = []
    for b in others:
        p = table[b // per] if b // per < len(table) else -1
        s = (q @ M[p, b % per]).max() if 0 <= p < M.shape[0] else -np.inf
        score.append(s if not np.isnan(s) else -np.inf)
    order = sorted(range(len(others)), key=lambda i: (-score[i], others[i]))
    if have <= first + last + top:
        return list(range(have))
    return sorted(always + [others[i] for i in order[:top] if score[i] > -np.inf])


def block_attention(q, K, V, M, table, cached: int, fresh: int, scale: float, block: int, first: int, last: int, top: int):
    hkv, page = K.shape[1], K.shape[2]
    G = q.shape[1] // hkv
    Kr, there = gather(K, table, cached + fresh)
    Vr, _ = gather(V, table, cached + fresh)
    t = np.arange(cached + fresh)
    out = []
    for i in range(fresh):
        row = []
        for h in range(hkv):
            ids = pick_blocks(q[i, h * G:h * G + G], M[:, h], table, block, page, cached + i, first, last, top)
            seen = there & (t <= cached + i) & np.isin(t // block, ids)
            row += [attend(q[i, g], Kr[h], Vr[h], seen, scale) for g in range(h * G, h * G + G)]
        out.append(row)
    return out
