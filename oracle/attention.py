"""Oracle of attention and its backward pass and of the gradients' norm, numpy in 64 bits, straight from the definitions in include/qrm.h: image by image,
head by head, only rows that are there."""
from __future__ import annotations

import numpy as np


def _lengths(lens, n, rows):
    return [rows] * n if lens is None else [int(min(max(int(x), 0), rows)) for x in lens]


def _heads(q, k, causal, q_len, k_len):
    """(image, head, key head, queries there, keys there, which query sees which key) of every image and head."""
    n, lq, heads, _ = q.shape
    lk, kv = k.shape[1], k.shape[2]
    ql, kl = _lengths(q_len, n, lq), _lengths(k_len, n, lk)
    for i in range(n):
        a, b = ql[i], kl[i]
        seen = np.ones((a, b), dtype=bool)
        if causal:
            seen = np.arange(b)[None] <= np.arange(a)[:, None] + b - a
        for h in range(heads):
            yield i, h, h // (heads // kv), a, b, seen


def attention(q, k, v, scale, causal=False, q_len=None, k_len=None):
    """q [N,Lq,heads,D], k, v [N,Lk,kv,D] -> o [N,Lq,heads,D], lse [N,heads,Lq], and the sums of P |v| (what a rounding of P moves o by)."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    n, lq, heads, _ = q.shape
    o, weight, lse = np.zeros_like(q), np.zeros_like(q), np.full((n, heads, lq), -np.inf)
    for i, h, g, a, b, seen in _heads(q, k, causal, q_len, k_len):
        rows = np.flatnonzero(seen.any(axis=1)) if b else np.zeros(0, dtype=int)
        if not rows.size:
            continue
        s = np.where(seen[rows], scale * (q[i, rows, h] @ k[i, :b, g].T), -np.inf)
        top = s.max(axis=1, keepdims=True)
        e = np.exp(s - top)
        total = e.sum(axis=1, keepdims=True)
        lse[i, h, rows] = (top + np.log(total))[:, 0]
        o[i, rows, h] = (e / total) @ v[i, :b, g]
        weight[i, rows, h] = (e / total) @ np.abs(v[i, :b, g])
    return o, lse, weight


def attention_backward(q, k, v, o, do, lse, scale, causal=False, q_len=None, k_len=None, score_off=0.0, product_off=0.0, half=0.0, sum_off=0.0):
    """-> (dq, dk, dv), and how far each may be off, (dq, dk, dv), where scores are off by score_off sum |q| |k| scale and relatively by it, products do v and
    do o by product_off of the sums of their magnitudes, P and dS by half after that, and long sums by sum_off of the sums of their magnitudes."""
    q, k, v, o, do = (np.asarray(t, dtype=np.float64) for t in (q, k, v, o, do))
    lse = np.asarray(lse, dtype=np.float64)
    grads, off = [np.zeros_like(t) for t in (q, k, v)], [np.zeros_like(t) for t in (q, k, v)]
    for i, h, g, a, b, seen in _heads(q, k, causal, q_len, k_len):
        rows = np.flatnonzero(seen.any(axis=1)) if b else np.zeros(0, dtype=int)
        if not rows.size:
            continue
        qi, ki, vi, oi, di, see = q[i, rows, h], k[i, :b, g], v[i, :b, g], o[i, rows, h], do[i, rows, h], seen[rows]
        s = scale * (qi @ ki.T)
        p = np.where(see, np.exp(np.where(see, s, 0.0) - lse[i, h, rows][:, None]), 0.0)
        dp, delta = di @ vi.T, (di * oi).sum(axis=1, keepdims=True)
        ds = p * (dp - delta)
        grads[0][i, rows, h] += scale * (ds @ ki)
        grads[1][i, :b, g] += scale * (ds.T @ qi)
        grads[2][i, :b, g] += p.T @ di
        rel = score_off * (1.0 + np.abs(s) + np.abs(lse[i, h, rows])[:, None] + scale * (np.abs(qi) @ np.abs(ki).T))
        p_off = p * rel
        ds_off = p_off * np.abs(dp - delta) + p * product_off * (np.abs(di) @ np.abs(vi).T + (np.abs(di) * np.abs(oi)).sum(axis=1, keepdims=True))
        ds_off += (half + sum_off) * np.abs(ds)
        off[0][i, rows, h] += scale * (ds_off @ np.abs(ki))
        off[1][i, :b, g] += scale * (ds_off.T @ np.abs(qi))
        off[2][i, :b, g] += (p_off + (half + sum_off) * p).T @ np.abs(di)
    return grads, off


def grad_norm(grads, max_norm, unscale=1.0):
    """-> norm, scale of a list of arrays (None: no gradient)."""
    total = sum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads if g is not None)
    norm = unscale * np.sqrt(total)
    return norm, unscale * (1.0 if norm <= max_norm else max_norm / norm)
