"""Oracles for drafted tokens: attention of a tree's nodes, verification, keeping.  TEST INFRASTRUCTURE ONLY.

Attention: row by row in float64 over the tokens that the node sees, those before the nodes and
the nodes of a set.  Verification: the rule as the proofs state it, node by node with explicit
lists: a node is accepted with probability min(1, r(t) / q(t)), r the target's probabilities at first
and, after each rejection, norm(max(r - q, 0)); the last token is drawn from r.
"""
from __future__ import annotations

import numpy as np


def tree_attention(q, k, v, sees, base, scale: float):
    """One request: q [n, H_q, D], k and v [L, H_kv, D] float64 (its L tokens); node i sees the tokens before `base`
    and base + j for j in sees[i] (those that exist).  Returns (O, lse, A, N), the last two as prompt_attention's."""
    n, Hq, D = q.shape
    L, H = k.shape[0], k.shape[1]
    O, A = np.zeros(q.shape), np.zeros(q.shape)
    lse, N = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    with np.errstate(invalid="ignore", over="ignore"):
        for i in range(n):
            at = sorted(set(range(max(0, min(base, L)))) | {base + j for j in sees[i] if 0 <= base + j < L})
            if not at:
                continue
            for h in range(Hq):
                kk, vv = k[at, h // (Hq // H)], v[at, h // (Hq // H)]
                s = scale * (kk @ q[i, h])
                N[i, h] = abs(scale) * float(np.max(np.abs(kk) @ np.abs(q[i, h])))
                m = s.max()
                e = np.exp(s - m)
                w = e / e.sum()
                O[i, h], A[i, h], lse[i, h] = w @ vv, w @ np.abs(vv), m + np.log(e.sum())
    return O, lse, A, N


class Border(ValueError):
    """A random number so near to a border that another order of the sums could choose otherwise."""


def verify(target, draft, tokens, parents, accept, final, margin=1e-12):
    """One request's nodes: target and draft [n, V] float64 (draft None: each token was certain), tokens, parents
    (node 0 the root) and random numbers as lists.  Returns (path, the last token).  A comparison whose sides are nearer than
    `margin` of the probabilities that they are differences of, and not equal (as where powers of two meet on purpose), raises
    Border; for the last token the share is at least that of V roundings."""
    n, V = target.shape

    def less(a, b, scale):
        if a != b and abs(a - b) <= margin * scale:
            raise Border(f"{a} and {b}")
        return a < b

    clean = lambda x: np.where(np.isfinite(x) & (x > 0), x, 0.0)
    path, cur = [0], 0
    r = clean(target[0])
    one = 1.0  # what r sums to: 1 by definition at first, and after each norm()
    left = 1.0  # what norm() has divided by: r * left is the difference of the rows
    i = 1
    while i < n:
        t = tokens[i]
        if parents[i] != cur or not 0 <= t < V:
            i += 1
            continue
        if draft is None:
            took = not (r[t] == 0 and _was_rejected(path, cur, i, tokens, parents)) and less(accept[i] * one, r[t], max(one, r[t]))
            if not took and not _was_rejected(path, cur, i, tokens, parents):
                one -= r[t]
                r = r.copy()
                r[t] = 0
        else:
            q = clean(draft[cur])
            took = less(accept[i] * q[t] * one, r[t], max(q[t], float(clean(target[cur])[t]) / left))
            if not took:
                r = np.maximum(r - q, 0)
                s = r.sum()
                r, one, left = (r / s, 1.0, left * s) if s > 0 else (r, 0.0, left)
        if took:
            cur = i
            path.append(i)
            r, one, left = clean(target[cur]), 1.0, 1.0
        i += 1
    if r.sum() == 0:
        r, left = clean(target[cur]), 1.0
    if r.sum() == 0:
        return path, -1
    cum = np.cumsum(r)
    aim = final * cum[-1]
    near = np.abs(cum[r > 0] - aim) <= max(margin, V * 2.0 ** -53 * (margin > 0)) * cum[-1] / left
    if np.any(near & (cum[r > 0] != aim)):
        raise Border(f"{final} of the last token")
    over = np.nonzero(cum > aim)[0]
    return path, int(over[0]) if len(over) else int(np.nonzero(r)[0][-1])


def _was_rejected(path, cur, i, tokens, parents):
    return any(parents[j] == cur and tokens[j] == tokens[i] for j in range(cur + 1, i))


def keep(cache, rows, cu, path, count):
    """On a kv_pages.Cache whose pools are [pages, 32, ...]: one token at a time."""
    ok = cache.named(rows)
    for i, r in enumerate(rows):
        n, m = cu[i + 1] - cu[i], int(count[i])
        if not ok[i] or not 0 <= m <= n or cache.lens[r] < n:
            continue
        mine = [int(x) for x in path[cu[i]:cu[i] + m]]
        if any(not 0 <= x < n for x in mine) or any(a >= b for a, b in zip(mine, mine[1:])):
            continue
        base = int(cache.lens[r]) - n
        written = {int(cache.table[r, h, (base + j) // 32]) for j, x in enumerate(mine) if x != j for h in range(cache.H)}
        if m < n and (base + m) % 32:  # (the page that the row would end inside, and be extended in)
            written |= {int(cache.table[r, h, (base + m) // 32]) for h in range(cache.H)}
        if any(0 <= p < len(cache.refs) and cache.refs[p] > 1 for p in written):  # (another row's as well)
            continue
        for j, x in enumerate(mine):
            for h in range(cache.H):
                a, b = (cache.table[r, h, (base + y) // 32] for y in (x, j))
                if all(0 <= p < len(cache.refs) for p in (a, b)):
                    for pool in cache.pools:
                        pool[b, (base + j) % 32] = pool[a, (base + x) % 32]
        for c in range(cache.pages(base + m), cache.pages(cache.lens[r])):
            for h in range(cache.H):
                p = cache.table[r, h, c]
                if 0 <= p < len(cache.refs):
                    cache.refs[p] -= 1
                cache.table[r, h, c] = -1
        cache.lens[r] = base + m
