"""Pages of a paged cache: extend, fork, shrink, free and compact on plain lists (oracle side).

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.
"""


class Model:
    def __init__(self, n_pages, page_tokens, max_seqs, width):
        self.T, self.width = page_tokens, width
        self.refs = [0] * n_pages
        self.table = [[-1] * width for _ in range(max_seqs)]
        self.lens = [0] * max_seqs
        self.status = 0                                          # the caller clears it
        self.refused = False

    def _free(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def _blame(self, code):
        self.status = self.status or code

    def extend(self, seqs, n_new):
        if self.refused and self.status:
            return
        self.refused, free, takes = True, self._free(), []
        for s, n in zip(seqs, n_new):
            if not 0 <= s < len(self.lens):
                continue
            if self.lens[s] + n > self.width * self.T:
                return self._blame(-2)
            takes += [(s, p) for p in range(-(-self.lens[s] // self.T), -(-(self.lens[s] + n) // self.T))]
        if len(takes) > len(free):
            return self._blame(-2)
        self.refused = False
        for (s, at), page in zip(takes, free):
            self.table[s][at], self.refs[page] = page, 1
        for s, n in zip(seqs, n_new):
            if 0 <= s < len(self.lens):
                self.lens[s] += n

    def fork(self, src, dst):
        """-> [(page copied, page it went to, tokens in it)]"""
        free, copies = self._free(), []
        if any(not 0 <= x < len(self.lens) for x in [*src, *dst]) or any(a == b or self.lens[b] for a, b in zip(src, dst)):
            self._blame(-3)
            return []
        lens = list(self.lens)
        if sum(lens[a] % self.T > 0 for a in src) > len(free):
            self._blame(-2)
            return []
        for a, b in zip(src, dst):
            full = lens[a] // self.T
            row = [-1] * self.width
            if lens[a]:
                row[:full] = self.table[a][:full]
            for p in row[:full]:
                self.refs[p] += 1
            if lens[a] % self.T:
                row[full] = free.pop(0)
                self.refs[row[full]] = 1
                copies.append((self.table[a][full], row[full], lens[a] % self.T))
            self.table[b], self.lens[b] = row, lens[a]
        return copies

    def free(self, seqs):
        for s in seqs:
            if not 0 <= s < len(self.lens):
                continue
            for p in self.table[s]:
                if p >= 0:
                    self.refs[p] -= 1
            self.table[s], self.lens[s] = [-1] * self.width, 0

    def shrink(self, seqs, n_drop, row_counts=()):
        """row_counts: the rows of a group of each row array."""
        if self.refused and self.status:
            return
        for s, n in zip(seqs, n_drop):
            if not 0 <= s < len(self.lens) or n <= 0:
                continue
            left = self.lens[s] - n
            if left < 0 or (left % self.T and self.refs[self.table[s][left // self.T]] != 1):
                return self._blame(-3)
            if any(left % r and left // r != self.lens[s] // r for r in row_counts):
                return self._blame(-3)
        for s, n in zip(seqs, n_drop):
            if not 0 <= s < len(self.lens) or n <= 0:
                continue
            for p in range(-(-(self.lens[s] - n) // self.T), -(-self.lens[s] // self.T)):
                self.refs[self.table[s][p]] -= 1
                self.table[s][p] = -1
            self.lens[s] -= n

    def compact(self):
        """-> [(page, where it went)]"""
        used = sum(r > 0 for r in self.refs)
        moves = list(zip([p for p, r in enumerate(self.refs) if r > 0 and p >= used], [p for p, r in enumerate(self.refs) if r == 0 and p < used]))
        to = dict(moves)
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
        return moves
