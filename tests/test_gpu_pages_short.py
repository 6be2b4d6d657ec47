"""Updates of page tables with too few pages, on the GPU: rows that get none keep their tokens."""
import pytest

torch = pytest.importorskip("torch")
from tests import pages_rules as pr  # noqa: E402
from tests import test_gpu_pages as tp  # noqa: E402

pytestmark = pytest.mark.gpu
ea = None
I32, BF = torch.int32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def library():
    global ea
    import paper_2502_12082_amd
    ea = tp.ea = paper_2502_12082_amd


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


class Server:
    """A cache of one layer, its tables, and the tokens that its rows should hold.  `many`: rows
    without tokens beside the others, as many as take the planner of large tables."""

    def __init__(self, page, pages, width, many):
        self.pool, self.many = pr.Pool(page, pages, width), 300 if many else 0
        self.cache = ea.paged_cache(pages, page, 1, 64)

    def step(self, parents, counts, by_rule=True):
        n = len(parents)
        parents, counts = parents + [-1] * self.many, counts + [0] * self.many
        pool = self.pool
        args = ints(pool.table), ints(pool.lengths()), ints(parents), ints(counts)
        table, lengths, missing = ea.cache_update(self.cache, *args)
        if by_rule:
            want = pr.update_by_rule(pool.table, pool.lengths(), parents, counts, pool.page, pool.pages)
            assert (table.tolist(), lengths.tolist(), missing.tolist()) == want[:3]
        new = pool.step(parents, counts, table.tolist(), lengths.tolist(), missing.tolist())
        if new:
            rows, positions, tokens = zip(*new)
            k = pr.token_rows(tokens).to(BF).cuda()
            ea.cache_append(self.cache, k, -k, ints(rows), ints(positions), table)
        held = [(r, at, t) for r, row in enumerate(pool.rows) for at, t in enumerate(row)]
        if held:
            rows, positions, tokens = zip(*held)
            want = pr.token_rows(tokens)
            k, v = ea.cache_read(self.cache, ints(rows), ints(positions), table)
            bad = ((k.float().cpu() != want) | (v.float().cpu() != -want)).flatten(1).any(1)
            assert not bad.any(), [held[i][:2] for i in bad.nonzero()[:, 0].tolist()]
        return lengths.tolist()[:n], missing.tolist()[:n]


@pytest.mark.parametrize("many", [False, True])
def test_the_longer_row_keeps_its_tokens(many):
    """Rows that share a page and both write to it, of different lengths, and no page is free."""
    # 18 and 20 tokens in the same two pages; the row that has room behind its tokens goes on
    s = Server(16, 2, 3, many)
    s.step([-1], [20])
    s.step([0, 0], [-2, 0])
    assert s.step([0, 1], [1, 1]) == ([18, 21], [1, 0])
    assert s.step([0, 1], [1, 1]) == ([18, 22], [1, 0])
    # the other way round, the lower row has more
    s = Server(16, 2, 3, many)
    s.step([-1], [20])
    s.step([0, 0], [0, -2])
    assert s.step([0, 1], [1, 1]) == ([21, 18], [0, 1])
    # the same length; then the rows change places
    s = Server(16, 2, 3, many)
    s.step([-1], [20])
    s.step([0, 0], [0, 0])
    assert s.step([0, 1], [1, 1]) == ([21, 20], [0, 1])
    assert s.step([1, 0], [1, 1]) == ([20, 22], [1, 0])
    # within the only page, and rows enough for a page's copy again when one ends
    s = Server(16, 1, 2, many)
    s.step([-1], [10])
    s.step([0, 0], [-2, 0])
    assert s.step([0, 1], [1, 1]) == ([8, 11], [1, 0])
    assert s.step([-1, 1], [0, 3]) == ([0, 14], [0, 0])


@pytest.mark.parametrize("many", [False, True])
def test_enough_pages(many):
    """With a page for the copy the lowest keeps the page, whichever has more."""
    s = Server(16, 3, 3, many)
    s.step([-1], [20])
    s.step([0, 0], [-2, 0])
    assert s.step([0, 1], [1, 1]) == ([19, 21], [0, 0])
    assert s.pool.table[0][:2] == [0, 1] and s.pool.table[1][:2] == [0, 2]


@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("first", range(0, 60, 15))
def test_short_pools(first, many):
    """Forks, growth and cut back rows in pools that are too small."""
    for seed in range(first, first + 15):
        page, pages, width, step, steps = pr.short_steps(seed, 8)
        s = Server(page, pages, width, many)
        for _ in range(steps):
            print(seed, flush=True)
            s.step(*step(len(s.pool.rows) - (s.many if len(s.pool.rows) > s.many else 0)))


@pytest.mark.parametrize("seed", [2, 19, 20])
def test_short_updates(seed):
    """Cases of test_update with too few pages: tables, copies and lengths by the rule.  (Of 19 that
    test holds the outcome in which row 92 writes to a place that row 248 has a token in.)"""
    page, pages, table, lengths, parents, counts = tp.table_case(seed)
    cache = torch.randint(0, 256, (2, pages, 1, 2, page // 16, 544), generator=torch.Generator().manual_seed(seed)).to(torch.uint8)
    t, l, m, copies = pr.update_by_rule(table, lengths, parents, counts, page, pages)
    assert any(n > 0 for n in m)
    got = cache.cuda()
    new = ea.cache_update(got, ints(table), ints(lengths), ints(parents), ints(counts))
    assert new[0].tolist() == t and new[1].tolist() == l and new[2].tolist() == m
    assert torch.equal(got.cpu(), tp.apply_copies(cache, copies))


# (rows, entries of each: planned by one workgroup, and from memory)
@pytest.mark.parametrize("rows,width", [(256, 40), (600, 40), (3000, 8), (40, 4000)])
def test_many_shared_pages(rows, width):
    """Many groups of rows that share their last page, of every length in it, and fewer pages than copies."""
    page, g = 16, torch.Generator().manual_seed(rows)
    table, lengths, at = [], [], 0
    while len(table) < rows:
        mine = [at, at + 1]
        at += 2
        for _ in range(min(rows - len(table), int(torch.randint(2, 9, (1,), generator=g)))):
            table.append(mine + [-1] * (width - 2))
            lengths.append(int(torch.randint(17, 32, (1,), generator=g)))
    pages = at + rows // 4
    parents = torch.randperm(rows, generator=g).tolist()
    counts = [1 if n % 50 else 0 for n in range(rows)]
    t, l, m, copies = pr.update_by_rule(table, lengths, parents, counts, page, pages)
    assert any(n > 0 for n in m) and copies
    cache = torch.randint(0, 256, (1, pages, 1, 2, 1, 544), generator=g).to(torch.uint8)
    got = cache.cuda()
    new = ea.cache_update(got, ints(table), ints(lengths), ints(parents), ints(counts))
    assert new[0].tolist() == t and new[1].tolist() == l and new[2].tolist() == m
    assert torch.equal(got.cpu(), tp.apply_copies(cache, copies))
    # no row writes where another has a token
    for r, n in enumerate(l):
        old = lengths[parents[r]]
        if n > old and old % page:
            p = t[r][old // page]
            assert all(l[o] <= old or t[o][old // page] != p for o in range(rows) if o != r), r
