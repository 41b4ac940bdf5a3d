"""What the page calls do to a table and its reference counts, one request after the other in plain Python."""
from __future__ import annotations

import numpy as np


class Pages:
    def __init__(self, n_seqs, row, n_pages, page_size):
        self.table = np.full((n_seqs, row), -1, dtype=np.int32)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.ps = page_size

    def _k(self, n):
        return -(-max(int(n), 0) // self.ps)

    def extend(self, seq, old, new):
        """(copy pairs, status)"""
        row, none = self.table.shape[1], [(-1, -1)] * len(seq)
        wanted, lacking = [], 0
        for i, b in enumerate(seq):
            if not 0 <= b < len(self.table) or new[i] <= max(old[i], 0):
                continue
            k0, k1 = self._k(old[i]), self._k(new[i])
            lacking += max(0, k1 - max(k0, row))
            if max(old[i], 0) % self.ps and k0 <= row:
                p = self.table[b, k0 - 1]
                if 0 <= p < len(self.refs) and self.refs[p] > 1:
                    wanted.append((i, b, k0 - 1, int(p)))
            wanted += [(i, b, k, -1) for k in range(k0, min(k1, row))]
        free = np.flatnonzero(self.refs <= 0)
        lacking += max(0, len(wanted) - len(free))
        if lacking:
            return none, [min(lacking, 2 ** 29), len(free)]
        for (i, b, k, src), p in zip(wanted, free):
            if src >= 0:
                none[i] = (src, int(p))
                self.refs[src] -= 1
            self.table[b, k] = p
            self.refs[p] = 1
        return none, [0, len(free) - len(wanted)]

    def fork(self, src, dst, n):
        for a, b, m in zip(src, dst, n):
            if not (0 <= a < len(self.table) and 0 <= b < len(self.table)) or a == b:
                continue
            for k in range(min(self._k(m), self.table.shape[1])):
                p = self.table[a, k]
                ok = 0 <= p < len(self.refs)
                self.table[b, k] = p if ok else -1
                if ok:
                    self.refs[p] += 1

    def truncate(self, seq, keep):
        for i, b in enumerate(seq):
            if not 0 <= b < len(self.table):
                continue
            for k in range(self._k(keep[i]) if keep is not None else 0, self.table.shape[1]):
                p = self.table[b, k]
                self.table[b, k] = -1
                if 0 <= p < len(self.refs):
                    self.refs[p] -= 1

    def compact(self):
        """(moves, status)"""
        used = np.flatnonzero(self.refs > 0)
        n = len(used)
        src = used[used >= n][::-1]
        dst = np.flatnonzero(self.refs[:n] <= 0)
        to = np.arange(len(self.refs))
        to[src] = dst
        live = (self.table >= 0) & (self.table < len(self.refs))
        self.table[live] = to[self.table[live]]
        self.refs[dst], self.refs[src] = self.refs[src], 0
        return list(zip(src.tolist(), dst.tolist())), [n, len(src)]
