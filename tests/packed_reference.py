"""Plain 64-bit statement of the 4-bit cache and of the page calls, value by value and page by page (numpy; shares no code with
the library).  Pool bytes: uint8 [pages][2][Hkv][P * (D / 2 + D / 16)]."""
from __future__ import annotations

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def e4m3_value(code):
    """Value of e4m3 codes (0x7f and 0xff: NaN)."""
    code = np.asarray(code).astype(np.int64)
    e, f = (code >> 3) & 15, code & 7
    v = np.where(e == 0, f / 8.0 * 2.0 ** -6, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((code & 127) == 127, np.nan, v)
    return np.where(code & 128, -v, v)


SCALES = e4m3_value(np.arange(127))  # 0 .. 448, ascending


def nearest(x, levels):
    """Index of the level nearest to x >= 0 (the even one of two equally near, the last for anything above)."""
    hi = np.clip(np.searchsorted(levels, x), 1, len(levels) - 1)
    lo = hi - 1
    a, b = x - levels[lo], levels[hi] - x
    return np.where((a < b) | ((a == b) & (lo % 2 == 0)), lo, hi)


def round_rows(x, scale):
    """float64 [..., D] -> value codes [..., D] and scale codes [..., D / 16]."""
    t = x.reshape(*x.shape[:-1], x.shape[-1] // 16, 16)
    f = nearest(np.abs(t).max(axis=-1) / scale / 6.0, SCALES)
    s = (SCALES[f] * scale)[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        n = nearest(np.where(s > 0, np.abs(t) / s, 0.0), LEVELS)
    n = np.where(s > 0, n + 8 * np.signbit(t), 0)
    return n.reshape(x.shape), f


def values(n, f, scale):
    v = np.where(n & 8, -1.0, 1.0) * LEVELS[n & 7]
    return (v.reshape(*v.shape[:-1], v.shape[-1] // 16, 16) * (e4m3_value(f) * scale)[..., None]).reshape(v.shape)


def put(pool, page, slot, which, P, n, f):
    """Writes one position's codes [Hkv][D] and scales [Hkv][D / 16] into the pool."""
    D = n.shape[-1]
    pool[page, which, :, slot * D // 2:(slot + 1) * D // 2] = n[:, 0::2] | n[:, 1::2] << 4
    at = P * D // 2 + slot * D // 16
    pool[page, which, :, at:at + D // 16] = f


def rows(pool, table, r, n, which, P, D, scale):
    """K (0) or V (1) of request r's positions 0 .. n - 1: float64 [n][Hkv][D]."""
    pos = np.arange(n)
    slab = pool[table[r, pos // P], which]  # [n][Hkv][bytes]
    slot = (pos % P)[:, None, None]
    i = np.arange(D)
    b = np.take_along_axis(slab, np.broadcast_to(slot * (D // 2) + i // 2, (n, slab.shape[1], D)), axis=2)
    code = (b >> (4 * (i % 2))) & 15
    k = np.arange(D // 16)
    f = np.take_along_axis(slab, np.broadcast_to(P * D // 2 + slot * (D // 16) + k, (n, slab.shape[1], D // 16)), axis=2)
    return values(code, f, scale)


def attention(K, V, q, ends, scale):
    """One request: K, V [L][Hkv][D], q [n][Hq][D], token i sees the first ends[i] keys -> out, lse, sum_j p_j |v_j|."""
    n, Hq, D = q.shape
    G = Hq // K.shape[1]
    out, mag, lse = np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    for i in range(n):
        L = int(ends[i])
        for h in range(Hq if L else 0):
            s = scale * (K[:L, h // G] @ q[i, h])
            e = np.exp(s - s.max())
            out[i, h], mag[i, h] = (e @ V[:L, h // G]) / e.sum(), (e @ np.abs(V[:L, h // G])) / e.sum()
            lse[i, h] = s.max() + np.log(e.sum())
    return out, lse, mag


def fork(ref, table, held, parent, length, need, P, out_blocks, fill):
    """-> ref_out, table_out (places behind a row's last hold `fill`), held_out, copy_src, copy_dst; None if pages run out."""
    n = len(parent)
    free = [p for p in range(len(ref)) if ref[p] == 0]
    new = np.array(ref)
    kids = {}
    for r in range(n):
        if parent[r] >= 0:
            kids.setdefault(int(parent[r]), []).append(r)
    for i in range(len(held)):
        for k in range(held[i]):
            new[table[i, k]] -= 1
    out = np.full((n, out_blocks), fill, np.int32)
    held_out, src, dst = np.zeros(n, np.int32), np.full(n, -1, np.int32), np.full(n, -1, np.int32)
    for r in range(n):
        p, full = int(parent[r]), int(length[r]) // P
        held_out[r] = -(-max(int(length[r]), int(need[r])) // P)
        for k in range(held_out[r]):
            page = int(table[p, k]) if p >= 0 and k < held[p] else -1
            mine = k < full or (page >= 0 and kids[p][0] == r and ref[page] == 1 and all(k >= length[c] // P for c in kids[p]))
            if not mine:
                if not free:
                    return None
                if k == full and length[r] % P:
                    src[r], dst[r] = page, free[0]
                page = free.pop(0)
            out[r, k] = page
            new[page] += 1
    return new, out, held_out, src, dst


def compact(ref, table, held, moves, fill):
    """-> ref_out, table_out, page_map, move_src, move_dst."""
    new, where = np.array(ref), np.arange(len(ref), dtype=np.int32)
    src, dst = np.full(moves, -1, np.int32), np.full(moves, -1, np.int32)
    holes, live = [p for p in range(len(ref)) if ref[p] == 0], [p for p in range(len(ref) - 1, -1, -1) if ref[p] > 0]
    for i, (h, p) in enumerate(zip(holes, live)):
        if i >= moves or h >= p:
            break
        src[i], dst[i], where[p], new[h], new[p] = p, h, h, ref[p], 0
    out = np.full(table.shape, fill, np.int32)
    for r in range(len(held)):
        out[r, : held[r]] = where[table[r, : held[r]]]
    return new, out, where, src, dst
