"""Plain fp64 oracle of the key/value cache: attention of drafted trees over a
paged cache with accumulated attention weight, appending, and eviction by that
weight. Written from the definitions, sequence by sequence and head by head.

A cache is a dict of arrays: k, v [n_pages, page, Hkv, d], page_table
[n_seq, max_pages], length, seen [n_seq], weight, pos [n_seq, Hkv, capacity].
"""
from __future__ import annotations

import numpy as np


def place(c, s, slot):
    """(page, row) of a slot, or None where the table has no page."""
    page = c["k"].shape[1]
    p = int(c["page_table"][s, slot // page])
    return (p, slot % page) if 0 <= p < c["k"].shape[0] else None


def ancestors(parent, n):
    """[n, n] bool: which drafted tokens each token sees."""
    sees = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while j >= 0:
            sees[i, j] = True
            up = j - 1 if parent is None else int(parent[j])
            j = up if 0 <= up < j else -1
    return sees


def tree_attention(c, q, k_new, v_new, tree_ptr, parent, scale, vote=None,
                   decay=1.0, max_tree=64, max_len=None):
    """dict of out [n_tok, Hq, d], lse [Hq, n_tok], weight, w_new [n_tok, Hkv]
    and, for tolerances, absv (the attention of |v|), absqk (the largest sum
    of |q||k| * scale of a row) [n_tok, Hq] and mass (the votes' sum without
    the old weight)."""
    n_tok, hq, d = q.shape
    hkv = c["k"].shape[2]
    group = hq // hkv
    out = np.full(q.shape, np.nan)
    absv = np.zeros(q.shape)
    absqk = np.zeros((n_tok, hq))
    lse = np.full((hq, n_tok), np.nan)
    weight = c["weight"].astype(np.float64).copy()
    absw = np.zeros_like(weight)
    w_new = np.full((n_tok, hkv), np.nan)
    vote = np.ones(n_tok) if vote is None else vote
    for s in range(len(tree_ptr) - 1):
        a = int(tree_ptr[s])
        n = min(int(tree_ptr[s + 1]) - a, max_tree)
        if n <= 0:
            continue
        ln = int(c["length"][s])
        if max_len is not None:
            ln = min(ln, max_len)
        at = [place(c, s, j) for j in range(ln)]
        slots = np.array([j for j in range(ln) if at[j] is not None], int)
        pages = np.array([at[j][0] for j in slots], int)
        offs = np.array([at[j][1] for j in slots], int)
        sees = ancestors(None if parent is None else parent[a:a + n], n)
        for g in range(hkv):
            k = c["k"][pages, offs, g].astype(np.float64)
            v = c["v"][pages, offs, g].astype(np.float64)
            total = np.zeros(len(slots))
            drafts = np.zeros(n)
            for h in range(g * group, (g + 1) * group):
                for i in range(n):
                    kk, vv = k, v
                    own = np.nonzero(sees[i])[0]
                    if k_new is not None:
                        kk = np.concatenate([k, k_new[a + own, g]])
                        vv = np.concatenate([v, v_new[a + own, g]])
                    with np.errstate(all="ignore"):
                        x = kk.astype(np.float64) @ q[a + i, h] * scale
                        top = x.max() if len(x) else -np.inf
                        if not len(x) or top == -np.inf and not np.isnan(
                                x).any():
                            out[a + i, h], lse[h, a + i] = 0.0, -np.inf
                            continue
                        e = np.exp(x - top)
                        p = e / e.sum()
                        out[a + i, h] = p @ vv
                        lse[h, a + i] = top + np.log(e.sum())
                        absv[a + i, h] = p @ np.abs(vv)
                        absqk[a + i, h] = scale * (
                            np.abs(kk) @ np.abs(q[a + i, h])).max()
                        if vote[a + i] != 0:
                            total += vote[a + i] * p[:len(slots)]
                            if k_new is not None:
                                drafts[own] += vote[a + i] * p[len(slots):]
            weight[s, g, :ln] *= decay
            weight[s, g, slots] += total
            absw[s, g, slots] = np.abs(total)
            w_new[a:a + n, g] = drafts
    return {"out": out, "lse": lse, "weight": weight, "w_new": w_new,
            "absv": absv, "absqk": absqk, "mass": absw}


def append(c, k_new, v_new, tok_ptr, max_new, accept=None, n_accept=None,
           w_new=None):
    """The cache afterwards (a new dict)."""
    r = {x: y.copy() for x, y in c.items()}
    cap = c["page_table"].shape[1] * c["k"].shape[1]
    for s in range(len(tok_ptr) - 1):
        a, rows = int(tok_ptr[s]), int(tok_ptr[s + 1] - tok_ptr[s])
        n = rows if n_accept is None else min(max(int(n_accept[s]), 0), rows)
        ln = int(c["length"][s])
        n = min(n, max_new, cap - ln)
        for i in range(n):
            j = i if accept is None else min(max(int(accept[a + i]), 0),
                                             rows - 1)
            p = place(c, s, ln + i)
            if p is not None:
                r["k"][p], r["v"][p] = k_new[a + j], v_new[a + j]
            r["weight"][s, :, ln + i] = 0 if w_new is None else w_new[a + j]
            r["pos"][s, :, ln + i] = c["seen"][s] + i
        r["length"][s] += n
        r["seen"][s] += n
    return r


def evict(c, budget, n_sink, n_recent, max_len=None):
    """The cache afterwards (a new dict)."""
    r = {x: y.copy() for x, y in c.items()}
    n_seq, hkv = c["weight"].shape[:2]
    for s in range(n_seq):
        ln = int(c["length"][s])
        if max_len is not None:
            ln = min(ln, max_len)
        if ln <= budget:
            continue
        for g in range(hkv):
            w = c["weight"][s, g, :ln].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            p = c["pos"][s, g, :ln].astype(np.int64)
            always = (p < n_sink) | (p >= int(c["seen"][s]) - n_recent)
            rank = sorted(range(ln), key=lambda j: (not always[j], -w[j], j)
                          if not always[j] else (False, 0.0, j))
            kept = set(rank[:budget])
            holes = [j for j in range(budget) if j not in kept]
            tails = [j for j in range(budget, ln) if j in kept]
            assert len(holes) == len(tails)
            for dst, src in zip(holes, tails):
                a, b = place(c, s, src), place(c, s, dst)
                if a is not None and b is not None:
                    r["k"][b[0], b[1], g] = c["k"][a[0], a[1], g]
                    r["v"][b[0], b[1], g] = c["v"][a[0], a[1], g]
                r["weight"][s, g, dst] = c["weight"][s, g, src]
                r["pos"][s, g, dst] = c["pos"][s, g, src]
        r["length"][s] = budget
    return r
