"""A step over a growing cache in 64 bits, from the definitions in the header: which rows a token has, norm and rotation, the
append, the attention of a draft tree, and what is kept of a draft.  numpy only; 8-bit and bf16 rows come as the numbers they stand for."""
from __future__ import annotations

import math

import numpy as np


def row_of(pair, t, n_rows, off=None, pages=None, page_rows=0):
    """Cache row of token t of a pair, None where the cache has none.  off [pairs] or pages [pairs][max_pages]."""
    if off is not None:
        first = int(off[pair])
        return first + t if first >= 0 and first + t < n_rows else None
    if t // page_rows >= pages.shape[1]:
        return None
    page = int(pages[pair, t // page_rows])
    return page * page_rows + t % page_rows if page >= 0 and (page + 1) * page_rows <= n_rows else None


def turned(x, norm, eps, table, pos, pairs):
    """Rows x [..., H, D] of tokens with positions pos [...]: normalised (norm [D] or None), rotated (table [n_pos][rot] or None)."""
    x = np.asarray(x, dtype=np.float64)
    if norm is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * np.asarray(norm, dtype=np.float64)
    if table is None:
        return x
    half = table.shape[1] // 2
    cos, sin = (np.asarray(table, dtype=np.float64)[pos][..., None, s] for s in (slice(0, half), slice(half, None)))
    a, b = (np.arange(half) * 2, np.arange(half) * 2 + 1) if pairs else (np.arange(half), np.arange(half) + half)
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def append(lens, cap, n_new, Hkv, row, ok_pos):
    """What an append does to the lengths: (new lens, {(pair, i): row}, pairs left alone).  row(pair, t) as row_of; ok_pos[b][i]."""
    out, rows, alone = [], {}, []
    for p, n0 in enumerate(int(x) for x in np.asarray(lens).reshape(-1)):
        n = int(n_new[p // Hkv])
        mine = [row(p, n0 + i) for i in range(n)] if n0 >= 0 and n0 + n <= int(np.asarray(cap).reshape(-1)[p]) else [None] * n
        if all(r is not None for r in mine) and all(ok_pos[p // Hkv][:n]):
            rows.update({(p, i): r for i, r in enumerate(mine)})
            out.append(n0 + n)
        else:
            alone.append(p)
            out.append(n0)
    return np.array(out, dtype=np.int32), rows, alone


def accept(lens, path, n_path, n_new, Hkv, row):
    """(new lens, {destination row: source row}, pairs left alone)."""
    out, moves, alone = [], {}, []
    for p, n0 in enumerate(int(x) for x in np.asarray(lens).reshape(-1)):
        b = p // Hkv
        n, kept, base = int(n_new[b]), int(n_path[b]), n0 - int(n_new[b])
        ok = 0 <= kept <= n and base >= 0 and all(0 <= int(j) < n for j in path[b][:kept])
        mine = [(row(p, base + i), row(p, base + int(path[b][i]))) for i in range(kept)] if ok else []
        if not ok or any(r is None for m in mine for r in m):
            alone.append(p)
            out.append(n0)
            continue
        moves.update(dict(mine))
        out.append(base + kept)
    return np.array(out, dtype=np.int32), moves, alone


def attend(q, k, v, lens, n_new, sees, scale, Hkv, row):
    """out [B][n][Hq][D], lse [B][n][Hq] and, for tolerances, the largest finite |v| that a column sees (a finite output is a mean of
    finite values, so that one bounds what rounded weights do to it) and the largest sum of |q_d k_d| * scale.
    sees(b, i, j): whether node i sees draft row j.  Nodes i >= n_new[b] are left NaN."""
    B, n, Hq, D = q.shape
    G = Hq // Hkv
    out, lse = np.full((B, n, Hq, D), np.nan), np.full((B, n, Hq), np.nan)
    v_top, s_top = np.zeros((B, n, Hq)), np.zeros((B, n, Hq))
    for b in range(B):
        m = int(n_new[b])
        for h in range(Hkv):
            length = max(int(np.asarray(lens).reshape(B, Hkv)[b, h]), 0)
            rows = [row(b * Hkv + h, t) for t in range(length)]
            there = np.array([r is not None for r in rows], dtype=bool)
            at = np.array([0 if r is None else r for r in rows], dtype=np.int64)
            kk, vv = k[at].astype(np.float64), v[at].astype(np.float64)
            draft = np.arange(length) - (length - m)
            for i in range(m):
                seen = there & np.array([j < 0 or sees(b, i, int(j)) for j in draft], dtype=bool)
                heads = slice(h * G, (h + 1) * G)
                if not seen.any():
                    out[b, i, heads], lse[b, i, heads] = 0.0, -math.inf
                    continue
                qq = q[b, i, heads].astype(np.float64)
                s = qq @ kk[seen].T * scale
                top = s.max(1, keepdims=True)
                w = np.exp(s - top)
                with np.errstate(invalid="ignore"):
                    out[b, i, heads] = w @ vv[seen] / w.sum(1, keepdims=True)
                lse[b, i, heads] = (top + np.log(w.sum(1, keepdims=True)))[:, 0]
                v_top[b, i, heads] = np.abs(vv[seen], where=np.isfinite(vv[seen]), out=np.zeros_like(vv[seen])).max()
                s_top[b, i, heads] = (np.abs(qq) @ np.abs(kk[seen]).T).max(1) * abs(scale)
    return out, lse, v_top, s_top
