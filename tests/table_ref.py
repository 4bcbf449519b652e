"""The pages of a worker's sequences by their definition, a sequence at a time on the host."""
import numpy as np


class Table:
    def __init__(self, S, width, page, pages, most):
        self.rows, self.length, self.refs = [[] for _ in range(S)], [0] * S, [0] * pages
        self.S, self.width, self.page, self.most = S, width, page, most

    def need(self, keys):
        return -(-keys // self.page)

    def advance(self, new, parent=None):
        """One step; returns (taken, copies, token_seq, token_pos)."""
        S, old = self.S, self.rows
        go = list(range(S)) if parent is None else [p if 0 <= p < S else None for p in parent]
        self.length = [0 if p is None else self.length[p] for p in go]
        self.length = [max(0, n + min(m, 0)) for n, m in zip(self.length, new)]
        self.rows = [[] if p is None else old[p][:self.need(n)] for p, n in zip(go, self.length)]
        self.count(old, -1)
        self.count(self.rows, 1)
        free = [p for p, r in enumerate(self.refs) if r == 0]
        sizes = [m if m > 0 and n + m <= self.width * self.page else 0 for n, m in zip(self.length, new)]
        plans, tokens, pages = [], 0, 0
        for s, m in enumerate(sizes):
            tokens += m
            if m == 0 or tokens > self.most:
                continue
            last = self.rows[s][-1] if self.length[s] % self.page else -1
            copy = last >= 0 and self.refs[last] > 1
            need = self.need(self.length[s] + m) - len(self.rows[s]) + copy
            pages += need
            if need == 0 or pages <= len(free):
                plans.append((s, m, need, copy))
        taken, copies, seq, pos, left = [0] * S, [[-1] * 3 for _ in range(S)], [], [], []
        for s, m, need, copy in plans:
            got, free = free[:need], free[need:]
            if copy:
                left.append(self.rows[s].pop())
                copies[s] = [left[-1], got[0], self.length[s] % self.page]
            self.rows[s] += got
            for p in got:
                self.refs[p] = 1
            seq += [s] * m
            pos += range(self.length[s], self.length[s] + m)
            taken[s] = m
            self.length[s] += m
        for p in left:
            self.refs[p] -= 1
        return taken, copies, seq, pos

    def count(self, rows, by):
        for row in rows:
            for p in row:
                self.refs[p] += by

    def padded(self):
        return np.array([row + [-1] * (self.width - len(row)) for row in self.rows])
