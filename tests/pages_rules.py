"""What an update of a page table has to give, also where the pool has too few pages, on the CPU."""
import random

import torch

from tests.pages_util import NUMBERS


def update_by_rule(table, lengths, parents, counts, page, pages):
    """(table, lengths, missing, copies) of an update, lists.  Of rows that all write to the page
    which they share one keeps it: the lowest, or where fewer pages are free than are
    needed, the one whose tokens end furthest into it (the lowest of such).  As many copies are
    made either way."""
    width, rows = len(table[0]), []
    for parent, count in zip(parents, counts):
        there = 0 <= parent < len(table)
        old = min(max(lengths[parent], 0), width * page) if there else 0
        new = max(0, old + count)
        fits = new <= width * page
        new = new if fits else old
        ids = list(table[parent][:-(-min(old, new) // page)]) if there else []
        writes = new > old and old % page != 0 and 0 <= ids[-1] < pages
        rows.append({"old": old, "new": new, "fits": fits, "ids": ids, "into": ids[-1] if writes else None})
    holders = {}
    for row in rows:
        for p in row["ids"]:
            if 0 <= p < pages:
                holders[p] = holders.get(p, 0) + 1
    writers = {}
    for r, row in enumerate(rows):
        if row["into"] is not None:
            writers.setdefault(row["into"], []).append(r)
    free = [p for p in range(pages) if p not in holders]

    def needs(first):
        """(whether it gets a copy, pages) of every row; first(r): the smallest keeps the page."""
        keeper = {p: min(w, key=first) for p, w in writers.items() if len(w) == holders[p]}
        out = []
        for r, row in enumerate(rows):
            copy = row["into"] is not None and keeper.get(row["into"]) != r
            out.append((copy, (-(-row["new"] // page) - len(row["ids"]) if row["new"] > row["old"] else 0) + copy))
        return out

    need = needs(lambda r: r)
    total = sum(n for _, n in need)
    if total > len(free):
        need = needs(lambda r: (-(rows[r]["old"] % page), r))
        assert sum(n for _, n in need) == total
    taken, missing, copies = 0, [], []
    for row, (copy, n) in zip(rows, need):
        mine, taken = free[taken:taken + n], taken + n
        missing.append(-1 if not row["fits"] else 0 if len(mine) == n else n)
        if missing[-1]:
            row["new"] = row["old"]
            continue
        if copy:
            copies.append((row["into"], mine[0]))
            row["ids"][-1] = mine.pop(0)
        row["ids"] += mine
    return ([row["ids"] + [-1] * (width - len(row["ids"])) for row in rows], [row["new"] for row in rows], missing,
            copies)


class Pool:
    """A pool of which every place holds the number of a token, and rows that know their tokens:
    what rows still hold is read back, whatever rule gave them their pages."""

    def __init__(self, page, pages, width):
        self.page, self.pages, self.width = page, pages, width
        self.places = {}  # (page, place in it): token
        self.table, self.rows, self.tokens = [[-1] * width], [[]], 0

    def lengths(self):
        return [len(r) for r in self.rows]

    def step(self, parents, counts, table, lengths, missing):
        """Rows after an update that gave these tables; returns the tokens to append, (row, position, token)."""
        rows, new = [], []
        for r, (parent, count) in enumerate(zip(parents, counts)):
            row = list(self.rows[parent]) if 0 <= parent < len(self.rows) else []
            if missing[r] == 0:
                row = row[:max(0, len(row) + count)] if count < 0 else row
                for _ in range(max(count, 0)):
                    new.append((r, len(row), self.tokens))
                    row.append(self.tokens)
                    self.tokens += 1
            assert lengths[r] == len(row), r
            rows.append(row)
        self.rows, self.table = rows, table
        return new

    def write(self, copies, new):
        """The pages of the update, on the CPU."""
        before = dict(self.places)
        for source, to in copies:
            for at in range(self.page):
                self.places[to, at] = before.get((source, at))
        for r, at, token in new:
            self.places[self.table[r][at // self.page], at % self.page] = token

    def lost(self):
        """(row, position) of tokens that a row has and its pages do not hold."""
        return [(r, at) for r, row in enumerate(self.rows) for at, token in enumerate(row)
                if self.places.get((self.table[r][at // self.page], at % self.page)) != token]


def short_steps(seed, steps=12):
    """(page, pages, width, rows of every step) of forks of different lengths in a pool that is too small."""
    rng = random.Random(seed)
    page, width = rng.choice([16, 32]), rng.choice([2, 3, 5])
    rows = rng.choice([2, 3, 6, 12])
    pages = rng.randrange(1, rows + 3)

    def step(now):
        """parents, counts for `now` rows."""
        n = rng.choice([now, rows, max(1, rows - 1)])
        favourite = rng.randrange(now)
        parents = [favourite if rng.random() < 0.4 else rng.randrange(-1, now) if rng.random() < 0.3 else r % now for r in range(n)]
        counts = [rng.choice([1, 1, 1, 0, 2, -1, -2, -3, -page, page // 2, page + 1]) for _ in range(n)]
        return parents, counts

    return page, pages, width, step, steps


def token_rows(tokens, d=64):
    """Keys of tokens' numbers that 4 bits hold as they are: the number's digits to the base of 8."""
    n = torch.tensor(tokens, dtype=torch.long).view(-1, 1)
    digit = (n >> 3 * torch.arange(8)) & 7
    x = torch.zeros(len(tokens), 1, d)
    x[:, 0, :8] = NUMBERS.float()[digit]
    x[:, 0, 8] = 6.0  # (the scale is 1)
    return x
