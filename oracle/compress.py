"""Compression of a growing cache in 64 bits, from the definitions in the header: the attention weight that every row gets, which rows stay,
and where they go.  numpy only; 8-bit and bf16 rows come as the numbers they stand for, row(pair, t) as oracle.step.row_of."""
from __future__ import annotations

import numpy as np


def attn_weights(q, k, lens, lse, old, scale, decay, n_new, tree, row, k_scale=None, fits=None):
    """New weights [n_rows] from `old`.  q [B, n, Hq, D], k [n_rows, D], lens [B][Hkv], lse [B, n, Hq], tree [B][n] words or None, n_new [B];
    fits(pair): whether a packed pair's run lies in the cache."""
    B, n, Hq, _ = q.shape
    Hkv = lens.shape[1]
    G = Hq // Hkv
    out = np.array(old, dtype=np.float64)
    for b in range(B):
        m = int(min(max(n_new[b], 0), n))
        for h in range(Hkv):
            pair, length = b * Hkv + h, int(max(lens[b, h], 0))
            if fits is not None and not fits(pair):
                continue
            at = [row(pair, t) for t in range(length)]
            t = np.array([x for x in range(length) if at[x] is not None], dtype=np.int64)
            rows = np.array([at[x] for x in t], dtype=np.int64)
            if not t.size:
                continue
            base = length - m
            w = np.where(t < base, decay * np.asarray(old, dtype=np.float64)[rows], 0.0) if decay else np.zeros(t.size)
            kk = np.asarray(k, dtype=np.float64)[rows] * (1.0 if k_scale is None else float(k_scale[h]))
            for i in range(m):
                word = (1 << (i + 1)) - 1 if tree is None else int(tree[b][i]) & (1 << 64) - 1
                sees = np.array([x < base or word >> int(x - base) & 1 for x in t], dtype=bool)
                for g in range(h * G, (h + 1) * G):
                    if lse[b, i, g] == -np.inf:
                        continue
                    z = scale * (kk[sees] * np.asarray(q[b, i, g], dtype=np.float64)).sum(-1)
                    w[sees] += np.exp(z - lse[b, i, g])
            out[rows] = w
    return out


def select(weights, lens, budget, shared, pool, sink, recent, max_keep, row):
    """(lists of the tokens that stay, per pair; their numbers, -1 where a list is longer than max_keep).  weights [n_rows], budget [B][Hkv] or [B]."""
    B, Hkv = lens.shape
    budget = np.asarray(budget).reshape(-1)
    lists = [None] * (B * Hkv)
    for group in range(B if shared else B * Hkv):
        pairs = range(group * Hkv, (group + 1) * Hkv) if shared else [group]
        ranked, stay = [], {}
        for p in pairs:
            n = max(int(lens.reshape(-1)[p]), 0)
            first = min(sink, n)
            end = max(first, n - min(recent, n))
            rows = {t: row(p, t) for t in range(n) if row(p, t) is not None}
            stay[p] = [t for t in rows if t < first or t >= end]

            def number(t):
                x = weights[rows[t]] if first <= t < end and t in rows else -np.inf
                return -np.inf if np.isnan(x) else float(x)

            ranked += [(-max(number(u) for u in range(max(first, t - pool // 2), min(end, t + pool // 2 + 1))), p, t) for t in rows if first <= t < end]
        room = max(0, int(budget[group]) - sum(len(x) for x in stay.values()))
        for _, p, t in sorted(ranked)[:room]:
            stay[p].append(t)
        for p in pairs:
            lists[p] = sorted(stay[p])
    return lists, np.array([len(x) if len(x) <= max_keep else -1 for x in lists], dtype=np.int32).reshape(B, Hkv)


def evict(lens, keep, n_keep, row, row_to=None, cap_to=None):
    """(new lens, {destination row: source row}, pairs left alone).  keep [B][Hkv][max_keep]; row_to and cap_to of another cache, None: in place."""
    lens, n_keep = (np.asarray(x).reshape(-1) for x in (lens, n_keep))
    keep = np.asarray(keep).reshape(lens.size, -1)
    to = row_to or row
    out, moves, alone = [], {}, []
    for p, n0 in enumerate(int(x) for x in lens):
        n = int(n_keep[p])
        ok = n0 >= 0 and 0 <= n <= keep.shape[1] and n <= (n0 if row_to is None else int(np.asarray(cap_to).reshape(-1)[p]))
        mine = [int(t) for t in keep[p][:n]] if ok else []
        ok = ok and all(0 <= t < n0 and row(p, t) is not None and to(p, i) is not None for i, t in enumerate(mine))
        ok = ok and (row_to is not None or all(x < y for x, y in zip(mine, mine[1:])))
        if ok:
            moves.update({to(p, i): row(p, t) for i, t in enumerate(mine)})
        else:
            alone.append(p)
        out.append(n if ok else n0 if row_to is None else 0)
    return np.array(out, dtype=np.int32), moves, alone
