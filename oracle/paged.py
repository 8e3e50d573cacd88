"""fp64 oracle of the paged cache: norm and rotation, and the bookkeeping of a pool written out one page after the other."""
from __future__ import annotations

import numpy as np

NONE = -1


def turned(x: np.ndarray, pos, inv_freq, weight=None, eps=1e-6, offset=0.0, scale=1.0, pairs=False):
    """Norm (with a weight) and rotation of rows x [n][H][D] at positions pos [n] -> (y, the sum of the magnitudes each entry is made of)."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * (np.asarray(weight, dtype=np.float64) + offset)
    y, mag = x.copy(), np.abs(x)
    r = 2 * len(inv_freq)
    for i, f in enumerate(inv_freq):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + r // 2)
        t = np.asarray(pos, dtype=np.float64)[:, None] * f
        y[..., a] = scale * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
        y[..., b] = scale * (x[..., b] * np.cos(t) + x[..., a] * np.sin(t))
        mag[..., a] = mag[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, mag


class Pool:
    """Tables, reference counts and page contents (data [slabs][pages][page][...])."""

    def __init__(self, table, refs, data, page):
        self.table, self.refs, self.data, self.page = np.array(table), np.array(refs), np.array(data), page
        self.bad_page = self.bad_length = self.no_pages = False

    def _row_ok(self, r, seen=()):
        ok = 0 <= r < len(self.table) and r not in seen
        self.bad_page |= not ok
        return ok

    def reserve(self, rows, lens, new_lens):
        P, N, cols = self.page, len(self.refs), self.table.shape[1]
        granted, todo, seen = [0] * len(rows), [], []
        for i, (r, a, b) in enumerate(zip(rows, lens, new_lens)):
            ok = self._row_ok(r, seen)
            seen.append(r)
            if not (0 <= a <= b <= cols * P):
                self.bad_length, ok = True, False
            if ok and b > a:
                for e in self.table[r, a // P:-(-b // P)]:
                    if e != NONE and not (0 <= e < N and self.refs[e] >= 1):
                        self.bad_page, ok = True, False
            if ok:
                todo.append(i)
        refs0 = self.refs.copy()

        def begun(i):                                   # the shared page that row i begins to write inside
            a, b = lens[i], new_lens[i]
            e = self.table[rows[i], a // P] if b > a and a % P else NONE
            return int(e) if e != NONE and refs0[e] > 1 else NONE

        writers = {}
        for i in todo:
            writers.setdefault(begun(i), []).append(i)
        keeps = {w[-1] for p, w in writers.items() if p != NONE and len(w) == refs0[p]}
        free = [p for p in range(N) if refs0[p] == 0]
        table0 = self.table.copy()
        out = False
        for i in todo:
            r, a, b = rows[i], lens[i], new_lens[i]
            need = []
            for j in range(a // P, -(-b // P)) if b > a else []:
                e = table0[r, j]
                if e == NONE or (refs0[e] > 1 and not (i in keeps and j == a // P)):
                    need.append(j)
            out |= len(need) > len(free)
            if out:
                self.no_pages = True
                continue
            granted[i] = 1
            for j in need:
                p, e = free.pop(0), table0[r, j]
                if e != NONE:
                    self.refs[e] -= 1
                    if j == a // P:
                        self.data[:, p, :a % P] = self.data[:, e, :a % P]
                self.refs[p] = 1
                self.table[r, j] = p
        return granted

    def fork(self, src, dst, lens):
        before, refs0, seen = self.table.copy(), self.refs.copy(), []

        def counted(e, refs):
            ok = 0 <= e < len(refs) and refs[e] >= 1
            self.bad_page |= not ok
            return ok

        for s, d, n in zip(src, dst, lens):
            ok = self._row_ok(d, seen) & self._row_ok(s)
            seen.append(d)
            if not 0 <= n <= self.table.shape[1] * self.page:
                self.bad_length, ok = True, False
            if not ok:
                continue
            for j in range(self.table.shape[1]):
                new = before[s, j] if j * self.page < n else NONE
                if new != NONE and not counted(new, refs0):
                    new = NONE
                if new != NONE:
                    self.refs[new] += 1
                if before[d, j] != NONE and counted(before[d, j], self.refs):
                    self.refs[before[d, j]] -= 1
                self.table[d, j] = new

    def release(self, rows, begin, end):
        for r, a, b in zip(rows, begin, end):
            if not self._row_ok(r):
                continue
            if a < 0:
                self.bad_length = True
                continue
            for j in range(self.table.shape[1]):
                e = self.table[r, j]
                if j * self.page >= a and (j + 1) * self.page <= b and e != NONE:
                    self.refs[e] -= 1
                    self.table[r, j] = NONE

    def compact(self):
        used = [p for p in range(len(self.refs)) if self.refs[p]]
        n = len(used)
        holes = [p for p in range(n) if not self.refs[p]]
        to = np.full(len(self.refs), NONE)
        for p in used:
            to[p] = p if p < n else holes.pop(0)
            if p >= n:
                self.data[:, to[p]] = self.data[:, p]
                self.refs[to[p]], self.refs[p] = self.refs[p], 0
        self.table = np.where(self.table >= 0, to[self.table], NONE)
        return to, n
