"""Plain 64-bit statement of cross attention, accumulated attention weights and cache eviction, request by request, over a
paged pool (numpy; shares no code with the library)."""
from __future__ import annotations

import numpy as np

from paper_2607_13095_b200 import workloads as wl


def rows(pool, table, r, n, which):
    """K (0) or V (1) of request r's positions 0 .. n - 1: float64 [n][Hkv][D] from bf16 bits [pages][2][Hkv][P][D]."""
    P = pool.shape[3]
    pos = np.arange(n)
    return wl.bits_to_f64(pool[table[r, pos // P], which, :, pos % P])


def cross_attention(pool, table, ctx, indptr, q, scale):
    """out, lse, and sum_j p_j |v_j| (what a relative error of the probabilities can move the output by)."""
    T, Hq, D = q.shape
    Hkv = pool.shape[2]
    G = Hq // Hkv
    out, mag, lse = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    for r in range(len(ctx)):
        a, b, L = int(indptr[r]), int(indptr[r + 1]), int(ctx[r])
        if a == b or L == 0:
            continue
        K, V, Q = rows(pool, table, r, L, 0), rows(pool, table, r, L, 1), wl.bits_to_f64(q[a:b])
        for h in range(Hq):
            S = scale * (Q[:, h] @ K[:, h // G].T)
            m = S.max(axis=1, keepdims=True)
            E = np.exp(S - m)
            den = E.sum(axis=1, keepdims=True)
            out[a:b, h] = (E @ V[:, h // G]) / den
            mag[a:b, h] = (E @ np.abs(V[:, h // G])) / den
            lse[a:b, h] = (m + np.log(den))[:, 0]
    return out, lse, mag


def self_lse(pool, table, ctx, indptr, q, scale):
    """lse of causal attention: token i of request r at position ctx + i, keys from the cache."""
    T, Hq, _ = q.shape
    G = Hq // pool.shape[2]
    lse = np.full((T, Hq), -np.inf)
    for r in range(len(ctx)):
        a, b, c = int(indptr[r]), int(indptr[r + 1]), int(ctx[r])
        if a == b:
            continue
        K, Q = rows(pool, table, r, c + b - a, 0), wl.bits_to_f64(q[a:b])
        seen = np.arange(c + b - a)[None, :] <= c + np.arange(b - a)[:, None]
        for h in range(Hq):
            S = np.where(seen, scale * (Q[:, h] @ K[:, h // G].T), -np.inf)
            m = S.max(axis=1)
            lse[a:b, h] = m + np.log(np.exp(S - m[:, None]).sum(axis=1))
    return lse


def attn_weights(pool, table, ctx, indptr, q, lse, scale, causal, decay, old):
    w = old.astype(np.float64).copy()
    Hkv = pool.shape[2]
    G = q.shape[1] // Hkv
    for r in range(len(ctx)):
        a, b, c = int(indptr[r]), int(indptr[r + 1]), int(ctx[r])
        n = b - a
        L = c + (n if causal else 0)
        w[r, :, :c] = decay * w[r, :, :c] if decay else 0.0
        w[r, :, c:L] = 0.0
        if n == 0 or L == 0:
            continue
        K, Q = rows(pool, table, r, L, 0), wl.bits_to_f64(q[a:b])
        for h in range(q.shape[1]):
            S = scale * (Q[:, h] @ K[:, h // G].T)
            seen = np.broadcast_to(lse[a:b, h][:, None] > -np.inf, S.shape).copy()
            if causal:
                seen &= np.arange(L)[None, :] <= c + np.arange(n)[:, None]
            with np.errstate(over="ignore", invalid="ignore"):
                w[r, h // G, :L] += np.where(seen, np.exp(S - lse[a:b, h].astype(np.float64)[:, None]), 0.0).sum(axis=0)
    return w


def evict_select(w, ctx, keep, max_keep, first, last):
    B, Hkv, _ = w.shape
    idx = np.full((B, Hkv, max_keep), -1, np.int32)
    kept = np.minimum(keep, ctx).astype(np.int32)
    for r in range(B):
        L = int(ctx[r])
        for kh in range(Hkv):
            v = w[r, kh, :L].astype(np.float64)
            v = np.where(np.isnan(v), -np.inf, v)
            # three classes: protected, ordinary, NaN; inside a class by weight, then by position
            cls = np.where(np.isnan(w[r, kh, :L]), 2, 1)
            j = np.arange(L)
            cls[(j < first) | (j >= L - last)] = 0
            v = np.where(cls == 1, v, 0.0)
            order = np.lexsort((j, -v, cls))
            idx[r, kh, : kept[r]] = np.sort(order[: kept[r]])
    return idx, kept


def evict_compact(pool, table, idx, kept, dst_table):
    """The pool after the move (a copy)."""
    P = pool.shape[3]
    out = pool.copy()
    for r in range(idx.shape[0]):
        for kh in range(idx.shape[1]):
            for i in range(int(kept[r])):
                j = int(idx[r, kh, i])
                out[dst_table[r, i // P], :, kh, i % P] = pool[table[r, j // P], :, kh, j % P]
    return out
