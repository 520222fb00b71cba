"""The book of pages, written out: which sequence holds which pages, one entry at a time.  Nothing of the library."""


def cdiv(a, b):
    return -(-a // b)


class Book:
    def __init__(self, pages, page_rows, slots, cols):
        self.refs, self.lens, self.rows = [0] * pages, [0] * slots, page_rows
        self.table, self.cols = [[0] * cols for _ in range(slots)], cols

    def copy(self):
        b = Book(len(self.refs), self.rows, len(self.lens), self.cols)
        b.refs, b.lens, b.table = list(self.refs), list(self.lens), [list(r) for r in self.table]
        return b

    def held(self, slot):
        return self.table[slot][:cdiv(self.lens[slot], self.rows)]

    def consistent(self):
        count = [0] * len(self.refs)
        for s in range(len(self.lens)):
            for p in self.held(s):
                count[p] += 1
        return count == self.refs

    def fork(self, src, dst):
        old, done = self.copy(), set()
        n = len(self.lens)
        for a, b in zip(src, dst):
            if not (0 <= a < n and 0 <= b < n) or b in done:
                continue
            done.add(b)
            if a == b:
                continue
            for p in old.held(b):
                self.refs[p] -= 1
            for p in old.held(a):
                self.refs[p] += 1
            self.lens[b] = old.lens[a]
            self.table[b][:len(old.held(a))] = old.held(a)

    def resize(self, slots, want):
        """(result, pairs of pages to copy); slots None: 0, 1, ..."""
        slots = range(len(want)) if slots is None else slots
        todo, done = [], set()
        for s, w in zip(slots, want):
            if 0 <= s < len(self.lens) and w >= 0 and s not in done:
                done.add(s)
                todo.append((s, w))
        if any(w > self.cols * self.rows for _, w in todo):
            return -1, []
        new = self.copy()
        for s, w in todo:
            for p in self.held(s)[cdiv(w, self.rows):]:
                new.refs[p] -= 1
        tails = {}                                     # pages that growing sequences would write into and others hold too
        for s, w in todo:
            old = self.lens[s]
            if w > old and old % self.rows:
                page = self.held(s)[-1]
                if new.refs[page] > 1:
                    tails.setdefault(page, []).append(s)
        takes = set()
        for page, who in tails.items():
            takes.update(who[1:] if len(who) == new.refs[page] else who)
        need = sum(max(cdiv(w, self.rows) - cdiv(self.lens[s], self.rows), 0) + (s in takes) for s, w in todo)
        free = [p for p, r in enumerate(new.refs) if r == 0]
        if need > len(free):
            return need - len(free), []
        pairs = []
        for s, w in todo:
            had, held = cdiv(self.lens[s], self.rows), cdiv(w, self.rows)
            if s in takes:
                old, page = new.table[s][had - 1], free.pop(0)
                new.refs[old] -= 1
                new.refs[page] = 1
                new.table[s][had - 1] = page
                pairs.append((old, page))
            for c in range(had, held):
                page = free.pop(0)
                new.refs[page] = 1
                new.table[s][c] = page
            new.lens[s] = w
        self.refs, self.lens, self.table = new.refs, new.lens, new.table
        return 0, pairs

    def compact(self):
        used = sum(1 for r in self.refs if r)
        movers = [p for p in range(used, len(self.refs)) if self.refs[p]]
        holes = [p for p in range(used) if not self.refs[p]]
        to = dict(zip(movers, holes))
        for s in range(len(self.lens)):
            for c in range(cdiv(self.lens[s], self.rows)):
                self.table[s][c] = to.get(self.table[s][c], self.table[s][c])
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        return used, list(to.items())
