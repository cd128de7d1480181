"""Plain 64-bit restatements of the paged-cache calls and of token sampling (host, numpy; shares no code with the library).

Written from the definitions in include/cascade.h: block tables and slots by walking the requests, attention row by row over
the keys a row sees, rotary embedding as complex multiplication, sampling by sorting.
"""
from __future__ import annotations

import numpy as np


def tables(new_len, kv_len, block_table, free_pages, count, page_size, n_tok, n_pages=None):
    """-> dict(table, free, count, kv, q_begin, slot, pos) of the next pass, or None where the call takes nothing."""
    new_len, kv_len = [int(x) for x in new_len], [int(x) for x in kv_len]
    table, free, count = np.array(block_table, np.int64), list(int(x) for x in free_pages), int(count)
    n_pages = len(free) if n_pages is None else n_pages
    pages = lambda n: -(-n // page_size)  # noqa: E731
    back = sum(pages(k) for n, k in zip(new_len, kv_len) if n < 0)
    need = sum(pages(k + n) - pages(k) for n, k in zip(new_len, kv_len) if n >= 0)
    if (min(kv_len) < 0 or any(k + max(n, 0) > table.shape[1] * page_size for n, k in zip(new_len, kv_len))
            or sum(max(n, 0) for n in new_len) > n_tok or not 0 <= count <= n_pages or count + back > n_pages
            or need > count + back):
        return None
    for r, n in enumerate(new_len):
        if n < 0:
            for j in range(pages(kv_len[r])):
                free[count] = int(table[r, j])
                count += 1
    kv, q_begin, slot, pos = [], [0], [], []
    for r, n in enumerate(new_len):
        if n < 0:
            kv.append(0)
            q_begin.append(len(slot))
            continue
        for j in range(pages(kv_len[r]), pages(kv_len[r] + n)):
            count -= 1
            table[r, j] = free[count]
        for x in range(kv_len[r], kv_len[r] + n):
            slot.append(int(table[r, x // page_size]) * page_size + x % page_size)
            pos.append(x)
        kv.append(kv_len[r] + n)
        q_begin.append(len(slot))
    rest = [-1] * (n_tok - len(slot))
    return dict(table=table, free=np.array(free), count=count, kv=np.array(kv), q_begin=np.array(q_begin),
                slot=np.array(slot + rest), pos=np.array(pos + rest))


def rotate(x, pos, base):
    """Rotary embedding of x [n,H,D] at positions pos [n]: element i and i + D/2 as one complex number."""
    D = x.shape[-1]
    z = np.asarray(x, np.float64)[..., : D // 2] + 1j * np.asarray(x, np.float64)[..., D // 2:]
    ang = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(D // 2) / D)[None, :]
    z = z * np.exp(1j * ang)[:, None, :]
    return np.concatenate([z.real, z.imag], -1)


def sees(x, n_keys, window, sinks):
    """Which of n_keys keys a row at position x sees."""
    j = np.arange(n_keys)
    ok = j <= x
    if window > 0:
        ok &= (j > x - window) | (j < sinks)
    return ok


def attention(q, k, v, window, sinks, scale):
    """One request: q [n,Hq,D] (its last n tokens), k, v [kv,Hkv,D] -> out [n,Hq,D], lse [n,Hq]."""
    n, Hq, D = q.shape
    kv, Hkv = k.shape[:2]
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    for i in range(n):
        ok = sees(kv - n + i, kv, window, sinks)
        if not ok.any():
            continue
        kk, vv = k[ok], v[ok]
        for h in range(Hq):
            s = kk[:, h // (Hq // Hkv)] @ q[i, h] * scale
            m = s.max()
            w = np.exp(s - m)
            out[i, h] = w @ vv[:, h // (Hq // Hkv)] / w.sum()
            lse[i, h] = m + np.log(w.sum())
    return out, lse


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """-> (token, prob, kept, gap): gap = how far u * total is from the nearest cumulative boundary, relative to total
    (and the nucleus' and min-p's decisions from theirs)."""
    row = np.asarray(row, np.float64).copy()
    V = len(row)
    row[np.isnan(row)] = -np.inf
    can = row > -np.inf
    if not can.any():
        return -1, 0.0, 0, 1.0
    m = row.max()
    if not temperature > 0:
        return int(np.argmax(row)), 1.0, 1, 1.0
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(row == m, 1.0, np.exp((row - m) / temperature)) if np.isfinite(temperature) else np.where(
            can, 1.0 if np.isfinite(m) else (row == m) * 1.0, 0.0)
    w[~can] = 0.0
    keep, gap = can.copy(), 1.0
    if 0 < top_k < V:
        keep &= row >= np.sort(row)[V - top_k]
    if top_p < 1:
        mass = w[keep].sum()
        values = np.unique(row[keep])[::-1]
        ahead, floor = 0.0, values[0]
        for x in values:
            gap = min(gap, abs(ahead / mass - top_p)) if x != values[0] else gap
            if x != values[0] and not ahead < top_p * mass:
                break
            floor = x
            ahead += w[keep & (row == x)].sum()
        keep &= row >= floor
    if min_p > 0:
        gap = min(gap, np.abs(w[keep & (row < m)] / min(min_p, 1.0) - 1).min(initial=1.0))
        keep &= w >= min(min_p, 1.0)
    ids = np.flatnonzero(keep)
    c = np.cumsum(w[ids])
    u = 0.0 if not u > 0 else min(float(u), 1 - 2.0 ** -24)
    i = min(int(np.searchsorted(c, u * c[-1], side="right")), len(ids) - 1)
    gap = min(gap, np.abs(c / c[-1] - u).min())
    return int(ids[i]), float(w[ids[i]] / c[-1]), len(ids), gap
