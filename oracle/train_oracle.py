"""Plain 64-bit restatements of a drafter's training operators (host, numpy; shares no code with the library).

Written from the definitions in include/cascade.h, position by position and row by row.
"""
from __future__ import annotations

import numpy as np

from oracle.paged_oracle import sees


def _entries(top, ids, V, temperature, target_lse):
    """(token, weight) of the stored logits that count, the target's log-sum-exp and their mass."""
    at = [(int(v), float(t) / temperature) for t, v in zip(top, ids) if 0 <= v < V]
    t = np.array([x for _, x in at], np.float64)
    if target_lse is None:
        if not len(t) or t.max() == -np.inf:
            return [], 0.0, 0.0
        lse = t.max() + np.log(np.exp(t - t.max()).sum())
    else:
        lse = float(target_lse)
    q = np.exp(t - lse)
    return [(v, w) for (v, _), w in zip(at, q)], lse, float(q.sum())


def distill_loss(draft, top, ids, target_lse=None, feat=None, seq=None, temperature=1.0, tau=0.5, c=2.0):
    """-> loss [K], saved [K,4], cosine [K] (NaN where none is looked at)."""
    draft = np.asarray(draft, np.float64)
    K, V = draft.shape
    loss, saved, cosine = np.zeros(K), np.zeros((K, 4)), np.full(K, np.nan)
    for k in range(K):
        if seq is not None and seq[k] < 0:
            continue
        w = 1.0
        if feat is not None and k + 1 < K and (seq is None or seq[k + 1] == seq[k]):
            a, b = np.asarray(feat[k], np.float64), np.asarray(feat[k + 1], np.float64)
            with np.errstate(invalid="ignore"):
                cosine[k] = a @ b / (np.sqrt(a @ a) * np.sqrt(b @ b))
            w = c if cosine[k] >= tau else 1.0
        x = draft[k] / temperature
        lse = x.max() + np.log(np.exp(x - x.max()).sum())
        entries, t_lse, mass = _entries(top[k], ids[k], V, temperature, None if target_lse is None else target_lse[k])
        loss[k] = w * sum(q * (lse - x[v]) for v, q in entries if q > 0)
        saved[k] = lse, t_lse, mass, w
    return loss, saved, cosine


def distill_grad(draft, top, ids, saved, grad_loss=None, scale=1.0, temperature=1.0):
    """The gradient from saved rows (lse, target lse, mass, weight)."""
    draft = np.asarray(draft, np.float64)
    K, V = draft.shape
    grad = np.zeros((K, V))
    for k in range(K):
        lse, t_lse, mass, w = (float(x) for x in saved[k])
        f = w * (1.0 if grad_loss is None else float(grad_loss[k])) * scale / temperature
        if f == 0:
            continue
        grad[k] = mass * np.exp(draft[k] / temperature - lse)
        for t, v in zip(top[k], ids[k]):
            if 0 <= v < V:
                grad[k, v] -= np.exp(float(t) / temperature - t_lse)
        grad[k] *= f
    return grad


def attention_grad(q, k, v, d_out, window, sinks, scale, out=None, lse=None):
    """One request: q, d_out [n,Hq,D], k, v [kv,Hkv,D] -> dq, dk, dv, each with the sum of its terms' sizes beside it.

    out, lse: those of the forward pass where the gradient is to be taken from them (else formed here)."""
    n, Hq, D = q.shape
    kv, Hkv = k.shape[:2]
    q, k, v, d_out = (np.asarray(t, np.float64) for t in (q, k, v, d_out))
    res = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)]
    size = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(k.shape)]
    for i in range(n):
        j = np.flatnonzero(sees(kv - n + i, kv, window, sinks))
        if not len(j):
            continue
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = k[j, g] @ q[i, h] * scale
            z = s.max() + np.log(np.exp(s - s.max()).sum()) if lse is None else float(lse[i, h])
            p = np.exp(s - z)
            o = p @ v[j, g] if out is None else np.asarray(out[i, h], np.float64)
            dp, delta = v[j, g] @ d_out[i, h], d_out[i, h] @ o
            ds = p * (dp - delta) * scale
            big = p * (np.abs(v[j, g]) @ np.abs(d_out[i, h]) + np.abs(d_out[i, h]) @ np.abs(o)) * scale
            res[0][i, h] = ds @ k[j, g]
            res[1][j, g] += ds[:, None] * q[i, h]
            res[2][j, g] += p[:, None] * d_out[i, h]
            size[0][i, h] = big @ np.abs(k[j, g])
            size[1][j, g] += big[:, None] * np.abs(q[i, h])
            size[2][j, g] += p[:, None] * np.abs(d_out[i, h])
    return res, size
