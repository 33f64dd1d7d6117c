"""The pages of a paged cache -- CPU ORACLE in plain Python (test infrastructure, not product): the same operations one
sequence, one page and one row after the other, on lists and numpy arrays."""
from __future__ import annotations


class Pages:
    def __init__(self, table, lens, refs, free, page_size):
        """table: list of rows, free: the free pages (the next one taken is the last)."""
        self.table, self.lens, self.refs, self.free = [list(r) for r in table], list(lens), list(refs), list(free)
        self.page = page_size

    def _valid(self, s):
        return 0 <= s < len(self.table)

    def fork(self, parents, children):
        empty = [n == 0 for n in self.lens]
        for i, (p, c) in enumerate(zip(parents, children)):
            if not self._valid(p) or not self._valid(c) or not empty[c] or c in parents or c in children[:i]:
                continue
            held = -(-self.lens[p] // self.page)
            self.table[c] = [x if n < held else -1 for n, x in enumerate(self.table[p])]
            for x in self.table[c]:
                if x >= 0:
                    self.refs[x] += 1
            self.lens[c] = self.lens[p]

    def extend(self, seqs, new_lens):
        """A page for every token that is new. -> (missing, moves), moves[i] = (src, dst, rows) or (-1, -1, 0)"""
        todo, seen, left = [], set(), dict()
        for i, (s, to) in enumerate(zip(seqs, new_lens)):
            if not self._valid(s) or s in seen:
                continue
            seen.add(s)
            to = min(max(to, self.lens[s]), len(self.table[s]) * self.page)
            n, entries = self.lens[s], []
            if to > n and n % self.page:
                at = n // self.page
                x = self.table[s][at]
                if x < 0:  # given back: the new rows on it need a page
                    entries.append((at, -1))
                else:
                    if self.refs[x] - left.get(x, 0) > 1:
                        entries.append((at, x))
                    left[x] = left.get(x, 0) + 1
            entries += [(p, -1) for p in range(-(-n // self.page), -(-to // self.page)) if self.table[s][p] < 0]
            todo.append((i, s, to, entries))
        moves = [(-1, -1, 0)] * len(seqs)
        lacking = sum(len(e) for _, _, _, e in todo) - len(self.free)
        if lacking > 0:
            return lacking, moves
        for i, s, to, entries in todo:
            for at, old in entries:
                new = self.free.pop()
                self.refs[new] = 1
                self.table[s][at] = new
                if old >= 0:
                    self.refs[old] -= 1
                    moves[i] = (old, new, self.lens[s] % self.page)
            self.lens[s] = max(to, self.lens[s])
        return 0, moves

    def release(self, seqs, first=None, last=None):
        before, freed = list(self.lens), []
        for i, s in enumerate(seqs):
            if not self._valid(s):
                continue
            n = before[s]
            lo, hi = max(first[i], 0) if first else 0, last[i] if last else n
            for p in range(-(-n // self.page)):
                if p * self.page >= lo and (min((p + 1) * self.page, n) <= hi if hi < n else True) and self.table[s][p] >= 0:
                    x, self.table[s][p] = self.table[s][p], -1
                    self.refs[x] -= 1
                    if self.refs[x] == 0:
                        freed.append(x)
            if hi >= n:
                self.lens[s] = min(self.lens[s], lo)
        self.free += sorted(freed)


def compact(k, place, lens, drafted, accepted, n_accepted):
    """Moves rows of k (numpy, in place); place(b, key) indexes a row for all heads. -> new lengths"""
    out = []
    for b, n in enumerate(lens):
        m = min(max(drafted[b], 0), n)
        base = n - m
        count = min(max(n_accepted[b], 0), m, len(accepted[b]))
        for i in range(count):
            node = min(max(accepted[b][i], i), m - 1)
            k[place(b, base + i)] = k[place(b, base + node)]
        out.append(base + count)
    return out
