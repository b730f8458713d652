"""A key-value cache in pages, from its definition: plain numpy in 64 bits, one sequence, head and row at a time.

Shares nothing with the library. Test infrastructure only."""
from __future__ import annotations

import numpy as np


def _place(table_row, P, i):
    return int(table_row[i // P]), i % P


def append(k, v, weight, pos, table, lens, seen, k_new, v_new, w_new=None):
    """k, v [n_pages][H][P][d]; weight, pos [n_pages][H][P] or None; k_new, v_new [S][H][n][d]. In place."""
    P, n = k.shape[2], k_new.shape[2]
    for s in range(len(lens)):
        for i in range(n):
            at = int(lens[s]) - n + i
            if at < 0:
                continue
            p, c = _place(table[s], P, at)
            if not 0 <= p < k.shape[0]:
                continue
            k[p, :, c], v[p, :, c] = k_new[s, :, i], v_new[s, :, i]
            if weight is not None:
                weight[p, :, c] = 0.0 if w_new is None else w_new[s, :, i]
                pos[p, :, c] = int(seen[s]) - n + i


def attend(k, v, weight, table, lens, q, decay=None):
    """q [S][n][Hq][d]. Returns out, lse; weight in place where decay is given. Tokens on pages outside the pool do not count."""
    n_pages, H, P, d = k.shape
    S, n, Hq, _ = q.shape
    G = Hq // H
    out, lse = np.zeros(q.shape), np.full(q.shape[:3], -np.inf)
    for s in range(S):
        T = int(lens[s])
        at = [_place(table[s], P, i) for i in range(T)]
        good = np.array([0 <= p < n_pages for p, _ in at], bool)
        pg = np.array([p if 0 <= p < n_pages else 0 for p, _ in at], int)
        sl = np.array([c for _, c in at], int)
        for h in range(H):
            got = np.zeros(T)
            for r in range(n):
                sees = good & (np.arange(T) <= T - n + r)
                if not sees.any():
                    continue
                kk, vv = k[pg[sees], h, sl[sees]], v[pg[sees], h, sl[sees]]
                for g in range(h * G, h * G + G):
                    x = kk @ q[s, r, g] / np.sqrt(d)
                    top = x.max()
                    if top == -np.inf:
                        continue
                    e = np.exp(x - top)
                    out[s, r, g] = (e / e.sum()) @ vv
                    lse[s, r, g] = top + np.log(e.sum())
                    got[sees] += e / e.sum()
            if decay is not None:
                old = weight[pg[good], h, sl[good]]
                weight[pg[good], h, sl[good]] = (0.0 if decay == 0 else decay * old) + got[good]
    return out, lse


def evict(k, v, weight, pos, table, lens, seen, keep, n_sink=0, n_recent=0):
    """In place, lens included. Weights are ordered as the 32-bit values they are held in."""
    n_pages, H, P, _ = k.shape
    for s in range(len(lens)):
        T = int(lens[s])
        if T <= keep:
            continue
        at = [_place(table[s], P, i) for i in range(T)]
        if any(not 0 <= p < n_pages for p, _ in at):
            continue
        for h in range(H):
            def order(i):
                p, c = at[i]
                fixed = pos[p, h, c] < n_sink or pos[p, h, c] >= int(seen[s]) - n_recent
                w = float(weight[p, h, c])
                return (0, 0.0, i) if fixed else (2, 0.0, i) if np.isnan(w) else (1, -w, i)
            stay = set(sorted(range(T), key=order)[:keep])
            free = [i for i in range(keep) if i not in stay]
            come = [i for i in range(keep, T) if i in stay]
            assert len(free) == len(come)
            for to, fr in zip(free, come):
                (pt, ct), (pf, cf) = at[to], at[fr]
                for x in (k, v, weight, pos):
                    x[pt, h, ct] = x[pf, h, cf]
        lens[s] = keep
