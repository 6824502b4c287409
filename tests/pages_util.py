"""The care of a cache's pages, written out in plain Python over lists: what the kernels have to do, one page at a time."""
import copy

SHORT, BAD_ROW, BAD_ID = 1, 2, 4


class State:
    def __init__(self, counts, tables, page, lens):
        self.counts, self.tables, self.page, self.lens = list(counts), [list(t) for t in tables], page, list(lens)
        self.wide = len(self.tables[0]) if self.tables else 0

    def pages(self, n):
        return -(-n // self.page)

    def fits(self, n):
        return 0 <= n <= self.wide * self.page

    def free_pages(self):
        return [p for p, c in enumerate(self.counts) if c == 0]

    def inside(self, page):
        return 0 <= page < len(self.counts)

    def fork(self, src, dst):
        """(moves, report)"""
        rows, free, flags, wanted = len(self.lens), self.free_pages(), 0, 0
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= s < rows and 0 <= d < rows and self.fits(self.lens[s]) and self.lens[d] == 0 and dst.count(d) == 1
            if not ok:
                flags |= BAD_ROW
        # (of a row listed twice one entry still counts as wanting: which is not said, so such lists are not compared in this)
        wanted = sum(1 for s, d in zip(src, dst) if 0 <= s < rows and 0 <= d < rows and self.fits(self.lens[s]) and self.lens[d] == 0
                     and self.lens[s] % self.page)
        if wanted > len(free):
            flags |= SHORT
        if flags:
            return [], [0, flags, len(free), wanted]
        before, moves = copy.deepcopy(self), []
        for s, d in zip(src, dst):
            n = before.lens[s]
            for j in range(n // self.page):
                page = before.tables[s][j]
                self.tables[d][j] = page
                if self.inside(page):
                    self.counts[page] += 1
                else:
                    flags |= BAD_ID
            if n % self.page:
                j, page = n // self.page, free.pop(0)
                flags |= 0 if self.inside(before.tables[s][j]) else BAD_ID
                self.tables[d][j] = page
                self.counts[page] = 1
                moves.append([before.tables[s][j], page])
            self.lens[d] = n
        return moves, [len(moves), flags, len(free), len(moves)]

    def grow(self, add):
        free, flags, wanted = self.free_pages(), 0, 0
        for n, a in zip(self.lens, add):
            if a > 0:
                if self.fits(n) and self.fits(n + a):
                    wanted += self.pages(n + a) - self.pages(n)
                else:
                    flags |= BAD_ROW
        if wanted > len(free):
            flags |= SHORT
        if flags:
            return [0, flags, len(free), wanted]
        for r, a in enumerate(add):
            if a > 0:
                for j in range(self.pages(self.lens[r]), self.pages(self.lens[r] + a)):
                    self.tables[r][j] = free.pop(0)
                    self.counts[self.tables[r][j]] = 1
                self.lens[r] += a
        return [wanted, 0, len(free), wanted]

    def free(self, rows):
        flags, freed = 0, 0
        for r in rows:
            if not 0 <= r < len(self.lens):
                flags |= BAD_ROW
                continue
            n, self.lens[r] = self.lens[r], 0
            if not self.fits(n):
                flags |= BAD_ROW
                continue
            for page in self.tables[r][: self.pages(n)]:
                if not self.inside(page) or self.counts[page] <= 0:
                    flags |= BAD_ID
                else:
                    self.counts[page] -= 1
                    freed += self.counts[page] == 0
        return [freed, flags, 0, 0]

    def compact(self, most):
        live = [p for p, c in enumerate(self.counts) if c]
        high = [p for p in live if p >= len(live)]
        low = [p for p in self.free_pages() if p < len(live)]
        assert len(high) == len(low)
        moves = [list(m) for m in zip(high, low)][:most]
        return moves, [len(moves), 0, len(self.counts) - len(live), len(high)]

    def remap(self, moves):
        to = {s: d for s, d in moves if self.inside(s) and self.inside(d)}
        for t, n in zip(self.tables, self.lens):
            for j in range(min(self.pages(max(n, 0)), self.wide)):
                t[j] = to.get(t[j], t[j])
        for s, d in to.items():
            self.counts[d], self.counts[s] = self.counts[s], 0


def random_state(rng, pages, rows, wide, page, fill, shared=0.3):
    """A state whose tables name about `fill` of the pool, rows sharing leading full pages with rows before them."""
    counts, order = [0] * pages, [int(x) for x in rng.permutation(pages)[: int(pages * fill)]]
    tables, lens = [[-5] * wide for _ in range(rows)], [0] * rows
    for r in range(rows):
        if rng.random() < 0.25:
            continue
        want, have = int(rng.integers(0, wide + 1)), []
        if r and rng.random() < shared:
            other = int(rng.integers(0, r))
            have = tables[other][: min(want, lens[other] // page)]
        while len(have) < want and order:
            have = have + [order.pop()]
        for p in have:
            counts[p] += 1
        tables[r][: len(have)] = have
        lens[r] = max(0, len(have) * page - (int(rng.integers(0, page)) if have else 0))
    return State(counts, tables, page, lens)
