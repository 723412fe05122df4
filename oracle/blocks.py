"""The book of a block cache in plain loops.

TEST INFRASTRUCTURE ONLY (see the package docstring).

table [rows, max_blocks] of block ids (-1: none), ref[b] entries that name b,
free: a list whose end is taken first, cache [blocks, bytes]; errors counts
what a call could not do.
"""
from __future__ import annotations

import numpy as np


class Book:
    def __init__(self, cache, bt, table, ref, free):
        self.cache, self.bt, self.table, self.ref, self.free = cache.copy(), bt, table.copy(), ref.copy(), list(free)
        self.errors = 0

    def _ok(self, b):
        return 0 <= b < len(self.ref)

    def _take(self):
        if not self.free:
            self.errors += 1
            return -1
        b = self.free.pop()
        self.ref[b] = 1
        return b

    def copy(self, src, dst):
        old = self.cache.copy()
        for s, d in zip(src, dst):
            if s == -1 or d == -1:
                continue
            if self._ok(s) and self._ok(d):
                self.cache[d] = old[s]
            else:
                self.errors += 1

    def fork(self, parents, children, lens):
        rows, width = self.table.shape
        for p, c, n in zip(parents, children, lens):
            if not (0 <= p < rows and 0 <= c < rows and p != c):
                self.errors += 1
                continue
            if not 0 <= n <= width * self.bt:
                self.errors += 1
                n = max(0, min(n, width * self.bt))
            full = n // self.bt
            row = np.full(width, -1, self.table.dtype)
            for j in range(full):
                b = self.table[p, j]
                if b == -1:
                    continue
                if self._ok(b):
                    row[j] = b
                    self.ref[b] += 1
                else:
                    self.errors += 1
            if n % self.bt and not self._ok(self.table[p, full]):
                self.errors += 1                         # nothing to copy
            elif n % self.bt:
                row[full] = self._take()
                if row[full] >= 0:
                    self.cache[row[full]] = self.cache[self.table[p, full]]
            self.table[c] = row

    def extend(self, rows, lens):
        for r, n in zip(rows, lens):
            if not 0 <= r < self.table.shape[0]:
                self.errors += 1
                continue
            if not 0 <= n <= self.table.shape[1] * self.bt:
                self.errors += 1
            for j in range(self.table.shape[1]):
                if j * self.bt < n and self.table[r, j] == -1:
                    self.table[r, j] = self._take()

    def release(self, rows):
        gone = []
        for r in rows:
            if not 0 <= r < self.table.shape[0]:
                self.errors += 1
                continue
            for j in range(self.table.shape[1]):
                b = self.table[r, j]
                self.table[r, j] = -1
                if b == -1:
                    continue
                if not self._ok(b) or self.ref[b] <= 0:
                    self.errors += 1
                    continue
                self.ref[b] -= 1
                if self.ref[b] == 0:
                    gone.append(int(b))
        self.free.extend(sorted(gone))

    def compact(self):
        """Returns the blocks' new ids (-1: free)."""
        live = [b for b in range(len(self.ref)) if self.ref[b] > 0]
        n = len(live)
        holes = [b for b in range(n) if self.ref[b] <= 0]
        new = np.full(len(self.ref), -1, np.int32)
        for b in live:
            new[b] = b if b < n else holes.pop(0)
        for b in live:
            if new[b] != b:
                self.cache[new[b]] = self.cache[b]
                self.ref[new[b]] = self.ref[b]
        self.ref[n:] = 0
        for r in range(self.table.shape[0]):
            for j in range(self.table.shape[1]):
                b = self.table[r, j]
                if b == -1:
                    continue
                if not self._ok(b):
                    self.errors += 1
                    continue
                self.errors += int(new[b] < 0)           # it named a free block
                self.table[r, j] = new[b]
        self.free = list(range(len(self.ref) - 1, n - 1, -1))
        return new
