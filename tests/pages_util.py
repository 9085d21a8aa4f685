"""What the calls that hand pages out have to do, in plain Python, one sequence after another."""
import numpy as np


class Pool:
    """table [S, max_pages], refs [n_pages] and the contents of each page in some layers, as numpy arrays."""

    def __init__(self, table, refs, page, layers=()):
        self.table, self.refs, self.page, self.layers = table.copy(), refs.copy(), page, [x.copy() for x in layers]

    def assign(self, source, lens):
        S, width = self.table.shape
        old = self.table.copy()
        for s in range(S):
            for c in range(width):
                p = -1
                if 0 <= source[s] < S and c * self.page < lens[s]:
                    p = old[source[s], c]
                self.table[s, c] = p if 0 <= p < len(self.refs) else -1
        for p in old.ravel():
            if 0 <= p < len(self.refs):
                self.refs[p] -= 1
        for p in self.table.ravel():
            if p >= 0:
                self.refs[p] += 1

    def reserve(self, start, count):
        S, width = self.table.shape
        was = self.refs.copy()
        free = [p for p in range(len(was)) if was[p] == 0]
        ok, closed, copies = [], False, []
        for s in range(S):
            if start[s] < 0 or count[s] < 0 or start[s] + count[s] > width * self.page:
                ok.append(0)
                continue
            span = range(start[s] // self.page, (start[s] + count[s] - 1) // self.page + 1) if count[s] else range(0)
            need = [c for c in span if not (0 <= self.table[s, c] < len(was)) or was[self.table[s, c]] != 1]
            closed = closed or len(need) > len(free)
            if need and closed:
                ok.append(0)
                continue
            ok.append(1)
            for c in need:
                p, new = self.table[s, c], free.pop(0)
                if 0 <= p < len(was):
                    copies.append((p, new))
                    self.refs[p] -= 1
                self.refs[new] = 1
                self.table[s, c] = new
        self.copy(copies)
        return ok

    def compact(self):
        live = [p for p in range(len(self.refs)) if self.refs[p] > 0]
        L = len(live)
        pairs = list(zip([p for p in live if p >= L], [p for p in range(L) if self.refs[p] <= 0]))
        self.copy(pairs)
        now = dict(pairs)
        for a, b in pairs:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = np.vectorize(lambda p: now.get(p, p), otypes=[np.int32])(self.table)
        return L

    def copy(self, pairs):
        for x in self.layers:
            was = x.copy()
            for a, b in pairs:
                x[b] = was[a]

    def consistent(self):
        n = np.bincount(self.table[self.table >= 0].ravel(), minlength=len(self.refs))
        return (n == self.refs).all()
