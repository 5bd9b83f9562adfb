"""A step of drafted decoding around the layers, by definition -- TEST INFRASTRUCTURE ONLY (the parity oracle of
``gdn_cache_tables``, ``gdn_draft_step`` and ``gdn_draft_verify``; only tests/ use it).

Page by page, token by token and probability by probability: nothing is shared with the HIP path.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

import oracle
from oracle.paged import spans


def cache_tables(lens, table, held, free, n_free, page, shared=None):
    """(table, held, free, n_free, missing) after a call: pages given back to the pool's end in order of sequence and entry,
    then the missing ones from there, all at once and in the pool's order."""
    table, held, free = np.array(table), [min(max(int(h), 0), np.shape(table)[1]) for h in held], np.array(free)
    n, width = table.shape
    pool = [int(x) for x in free[:min(max(int(n_free), 0), len(free))]]
    want = []
    for i in range(n):
        need = min(-(-max(int(lens[i]), 0) // page), width)
        if shared is not None:
            need = max(need, min(int(shared[i]), held[i]))
        for e in range(need, held[i]):
            pool.append(int(table[i, e]))
            free[len(pool) - 1] = table[i, e]
            table[i, e] = -1
        want += [(i, e) for e in range(held[i], need)]
        held[i] = min(held[i], need)
    got = min(len(want), len(pool))
    taken, pool = pool[len(pool) - got:], pool[:len(pool) - got]
    for k, (i, e) in enumerate(want):
        table[i, e] = taken[k] if k < got else -1
        held[i] += k < got
    return table, np.array(held), free, len(pool), len(want) - got


def step_maps(lens, table, n_pages, page, rows, new=None):
    """(offsets, positions, slots) of a step's rows; ``new`` None: rows / n each."""
    n, width = np.shape(table)
    cu = [0]
    for i in range(n):
        cu.append(min(cu[-1] + (rows // n if new is None else max(int(new[i]), 0)), rows))
    pos, slots = np.zeros(rows, dtype=np.int64), np.full(rows, -1, dtype=np.int64)
    for i in range(n):
        for t in range(cu[i], cu[i + 1]):
            pos[t] = max(int(lens[i]), 0) - cu[i + 1] + t
            if 0 <= pos[t] < width * page and 0 <= table[i][pos[t] // page] < n_pages:
                slots[t] = int(table[i][pos[t] // page]) * page + pos[t] % page
    return np.array(cu), pos, slots


def draft_step(q, k, v, g, beta, S, keep=None, cu=None, **kw):
    """(o, S after the first keep[s] tokens of each sequence); rows of no sequence are NaN in o."""
    v = np.asarray(v, dtype=np.float64)
    o, S_new = np.full(v.shape, np.nan), np.array(S, dtype=np.float64)
    B, T, H, dv = v.shape
    flat = [np.asarray(x, dtype=np.float64).reshape(B * T, *np.shape(x)[2:]) for x in (q, k, v, g, beta)]
    for s, (at, m) in enumerate(spans(B, T, cu)):
        kept = m if keep is None else min(max(int(keep[s]), 0), m)
        for count, out in ((m, True), (kept, False)):
            if count:
                part = [x[None, at:at + count] for x in flat]
                y, state = oracle.recurrence_ex(*part, S0=np.asarray(S, dtype=np.float64)[s:s + 1], **kw)
                if out:
                    o.reshape(B * T, H, dv)[at:at + m] = y[0]
                else:
                    S_new[s] = state[0]
    return o, S_new


def verify(p, q, drafts, lens, u):
    """(tokens [n, m + 1], counts [n]) in exact rationals."""
    n, rows, V = np.shape(p)
    m = rows - 1
    clean = lambda x: Fraction(float(x)) if np.isfinite(x) and x > 0 else Fraction(0)   # noqa: E731
    tokens, counts = np.full((n, m + 1), -1), np.zeros(n, dtype=int)
    for s in range(n):
        len_s = m if lens is None else min(max(int(lens[s]), 0), m)
        j = 0
        while j < len_s:
            x = int(drafts[s][j])
            if not 0 <= x < V:
                break
            qx = Fraction(1) if q is None else clean(q[s][j][x])
            if not (np.isfinite(u[s][j]) and Fraction(float(u[s][j])) * qx < clean(p[s][j][x])):
                break
            tokens[s, j] = x
            j += 1
        target = [clean(x) for x in p[s][j]]
        w = target
        if j < len_s:
            less = [clean(x) for x in q[s][j]] if q is not None else [Fraction(int(x == drafts[s][j])) for x in range(V)]
            w = [max(a - b, Fraction(0)) for a, b in zip(target, less)]
        w = w if sum(w) > 0 else target
        draw = u[s][m]
        goal = (Fraction(float(draw)) if draw > 0 else Fraction(0)) * sum(w)   # (NaN: 0)
        run, best = Fraction(0), -1
        for x in range(V):
            if w[x] > 0:
                best = x
                run += w[x]
                if run > goal:
                    break
        tokens[s, j] = best
        counts[s] = j + 1
    return tokens, counts
