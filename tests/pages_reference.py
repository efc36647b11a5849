"""Edits of a paged cache's tables in plain Python, from the rules of
include/agft_pages.h, on top of kv_reference.Node.  One request and one page at a
time; no code shared with the package."""
from kv_reference import Node


class Pages(Node):
    """A node whose pages may have several owners."""

    def __init__(self, *args):
        super().__init__(*args)
        self.owners = [0] * self.P

    @property
    def extra(self):
        return sum(self.owners)

    def plan(self, add, max_tokens):
        """As a node's, but no request ends while a page has several owners."""
        stuck = [a < 0 and self.extra > 0 for a in add]
        want = super().plan([0 if s else a for a, s in zip(add, stuck)], max_tokens)
        want["counters"][3] += sum(stuck)
        return want

    def fork(self, src, dst, tokens):
        table, lengths, granted, moves, asked, shared = self.table.copy(), list(self.lengths), [], [], 0, []
        for a, b, t in zip(src, dst, tokens if tokens is not None else [1 << 30] * len(src)):
            t = min(t, self.lengths[a]) if 0 <= a < self.R and 0 <= b < self.R else 0
            if a == b or dst.count(b) > 1 or (0 <= b < self.R and self.lengths[b]) or t < 0:
                t = 0
            asked += t % self.page > 0
            if t > 0 and t % self.page > 0 and asked > self.free:
                t = 0
            granted.append(t)
            moves.append([-1, -1])
            full = t // self.page
            if t:
                lengths[b] = t
                table[b, :full] = self.table[a, :full]
                shared += [int(x) for x in self.table[a, :full]]
            if t % self.page:
                moves[-1] = [int(self.table[a, full]), self.ring[(self.head + asked - 1) % self.P]]
                table[b, full] = moves[-1][1]
        taken = sum(m[0] >= 0 for m in moves)
        self.table = table
        return dict(kind="fork", lengths=lengths, granted=granted, moves=moves, shared=shared,
                    counters=[(self.head + taken) % self.P, self.free - taken, self.extra + len(shared),
                              granted.count(0), taken, 0, len(moves), 1])

    def trim(self, keep):
        lengths, refused, gone = [], 0, []
        for i, k in enumerate(keep):
            n = self.lengths[i]
            if not 0 <= k < n:
                k = n
            if k < n and k % self.page and self.owners[int(self.table[i, k // self.page])] > 0:
                k, refused = n, refused + 1
            lengths.append(k)
            gone += [int(self.table[i, m]) for m in range(self._pages(k), self._pages(n))]
        back = [p for m, p in enumerate(gone) if gone.count(p) == self.owners[p] + 1 and p not in gone[m + 1:]]
        for m, p in enumerate(back):
            self.ring[(self.head + self.free + m) % self.P] = p
        return dict(kind="trim", lengths=lengths, gone=gone, moves=[],
                    counters=[self.head, self.free + len(back), self.extra - (len(gone) - len(back)), refused, 0,
                              len(back), 0, 2])

    def compact(self):
        free = {self.ring[(self.head + m) % self.P] for m in range(self.free)}
        n = self.P - self.free
        moves = [list(m) for m in zip([p for p in range(n, self.P) if p not in free], [p for p in range(n) if p in free])]
        return dict(kind="compact", lengths=list(self.lengths), moves=moves,
                    counters=[n % self.P, self.free, self.extra, 0, 0, 0, len(moves), 3])

    def copy(self, edit):
        for a, b in edit["moves"]:
            if a >= 0:
                self.codes[b], self.exps[b] = self.codes[a], self.exps[a]

    def commit_edit(self, edit):
        if edit["kind"] == "fork":
            for p in edit["shared"]:
                self.owners[p] += 1
        elif edit["kind"] == "trim":
            for p in edit["gone"]:
                self.owners[p] = max(0, self.owners[p] - 1)
        else:
            to = dict(edit["moves"])
            for i in range(self.R):
                for m in range(self._pages(self.lengths[i])):
                    self.table[i, m] = to.get(int(self.table[i, m]), int(self.table[i, m]))
            for a, b in edit["moves"]:
                self.owners[b], self.owners[a] = self.owners[a], 0
            self.ring = list(range(self.P))
        self.lengths = list(edit["lengths"])
        self.head, self.free = edit["counters"][:2]
        assert self.extra == edit["counters"][2]
