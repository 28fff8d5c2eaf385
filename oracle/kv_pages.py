"""Oracle for the pages of a paged cache.  TEST INFRASTRUCTURE ONLY.

The rules, one page at a time, on plain Python lists and numpy arrays: extend takes the
lowest free pages, fork shares whole pages and copies a part page, free gives up, compact
moves the live pages at or above their number into the holes below it.
"""
from __future__ import annotations

import numpy as np

PT = 32


class Cache:
    def __init__(self, table, lens, refs, pools=()):
        self.table, self.lens, self.refs = np.array(table), np.array(lens), np.array(refs)
        self.pools = [np.array(p) for p in pools]
        self.R, self.H, self.pph = self.table.shape

    def pages(self, n: int) -> int:
        return min(-(-max(int(n), 0) // PT), self.pph)

    def free_pages(self):
        return [p for p in range(len(self.refs)) if self.refs[p] <= 0]

    def named(self, rows):
        seen, out = set(), []
        for r in rows:
            out.append(0 <= r < self.R and r not in seen)
            seen.add(r)
        return out

    def extend(self, rows, new_lens):
        ok = self.named(rows)
        free, take = self.free_pages(), []
        for i, (r, n) in enumerate(zip(rows, new_lens)):
            if ok[i] and self.lens[r] < n <= self.pph * PT:
                take += [(r, h, c) for h in range(self.H) for c in range(self.pages(self.lens[r]), self.pages(n))]
            else:
                ok[i] = False
        if len(take) > len(free):
            return 0, len(take) - len(free)
        for (r, h, c), p in zip(take, free):
            self.table[r, h, c], self.refs[p] = p, 1
        for i, r in enumerate(rows):
            if ok[i]:
                self.lens[r] = new_lens[i]
        return len(take), 0

    def release(self, r):
        for h in range(self.H):
            for c in range(self.pages(self.lens[r])):
                p = self.table[r, h, c]
                if 0 <= p < len(self.refs):
                    self.refs[p] -= 1

    def fork(self, src, dst):
        ok = [n and 0 <= s < self.R and s != d for n, s, d in zip(self.named(dst), src, dst)]
        free = self.free_pages()
        need = sum(self.H for i, s in enumerate(src) if ok[i] and self.lens[s] % PT)
        if need > len(free):
            return 0, need - len(free)
        new, took = [], 0
        for i, s in enumerate(src):
            if not ok[i]:
                continue
            row = np.full((self.H, self.pph), -1, self.table.dtype)
            whole = int(self.lens[s]) // PT
            for h in range(self.H):
                for c in range(whole):
                    row[h, c] = self.table[s, h, c]
                    if 0 <= row[h, c] < len(self.refs):
                        self.refs[row[h, c]] += 1
                if self.lens[s] % PT:
                    p = free[took]
                    took += 1
                    row[h, whole], self.refs[p] = p, 1
                    for pool in self.pools:
                        pool[p] = pool[self.table[s, h, whole]]
            new.append((dst[i], row, int(self.lens[s])))
        for d, row, n in new:
            self.release(d)
        for d, row, n in new:
            self.table[d], self.lens[d] = row, n
        return need, 0

    def free(self, rows):
        for ok, r in zip(self.named(rows), rows):
            if ok:
                self.release(r)
                self.table[r], self.lens[r] = -1, 0

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] <= 0]
        moved = [p for p in live if p >= n]
        to = dict(zip(moved, holes))
        for a, b in to.items():
            for pool in self.pools:
                pool[b] = pool[a]
            self.refs[b], self.refs[a] = self.refs[a], 0
        for e in np.ndindex(self.table.shape):
            self.table[e] = to.get(int(self.table[e]), self.table[e])
        return len(holes), n
