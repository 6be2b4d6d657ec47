"""A cache in pages and in 4 bits as a server uses it: prompts, decoding steps, beams and
drafts, with everything on the device, eager and in a graph."""
import pytest

torch = pytest.importorskip("torch")
from tests import pages_util as pu  # noqa: E402
from tests.layer_util import check, packed64  # noqa: E402

pytestmark = pytest.mark.gpu
ea = None
I32, BF, F32 = torch.int32, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    global ea
    import paper_2502_12082_amd
    ea = paper_2502_12082_amd


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


class ByHand:
    """Rows of keys and values, as lists of tokens, and what a step gives."""

    def __init__(self, layers, hk, d):
        self.rows, self.layers, self.hk, self.d = [], layers, hk, d

    def step(self, parents, counts, k, v):
        """k, v [layers, tokens, hk, d] of the new tokens, row by row."""
        rows, at = [], 0
        held = [pu.unpack(*pu.pack(t)) for t in (k, v)]
        for p, n in zip(parents, counts):
            row = list(self.rows[p]) if 0 <= p < len(self.rows) else []
            if n < 0:
                row = row[:n]
            for _ in range(max(n, 0)):
                row.append((held[0][:, at], held[1][:, at]))
                at += 1
            rows.append(row)
        self.rows = rows

    def check(self, cache, table, lengths, q, o, layer):
        page = 16 * cache.shape[4]
        assert lengths.tolist() == [len(r) for r in self.rows]
        # the values that the pages hold, and attention over them
        vals = pu.values(cache[layer])
        t = table.cpu()
        for r, row in enumerate(self.rows):
            keys, values, there = pu.keys_of(vals, t, r, len(row), page)
            assert there.all()
            for at, (k, v) in enumerate(row):
                assert torch.equal(keys[at], k[layer]) and torch.equal(values[at], v[layer]), (r, at)
        want, off = pu.paged64(q, vals, t, lengths.cpu(), None, page, 1.5, self.d ** -0.5)
        check("together", o, want, 0.0, off)


def new_tokens(lengths, counts):
    """(rows, positions) of the tokens that rows of these new lengths gained."""
    rows = [r for r, n in enumerate(counts) for _ in range(max(n, 0))]
    positions = [p for n, c in zip(lengths, counts) for p in range(n - max(c, 0), n)]
    return ints(rows), ints(positions)


@pytest.mark.parametrize("dtype,d,page", [(BF, 128, 16), (F32, 64, 32)])
def test_serving_steps(dtype, d, page):
    layers, hk, hq, width, pages = 2, 2, 4, 12, 60
    g = torch.Generator().manual_seed(d)
    cache = ea.paged_cache(pages, page, hk, d, layers)
    assert ea.paged_cache(pages, page, hk, d).shape == cache.shape[1:]
    table, lengths = torch.full((1, width), -1, dtype=I32, device="cuda"), ints([0])
    hand = ByHand(layers, hk, d)
    steps = [
        ([-1, -1, -1], [page + 3, 2 * page, 5]),      # prompts
        ([0, 1, 2], [1, 1, 1]),                       # a step
        ([0, 0, 0, 1, 2], [1, 1, 1, 1, 0]),           # the first goes on three times, the last waits
        ([2, 0, 0, 3, 4], [1, 2, 1, -page, 1]),       # beams change places, one row drops a draft
        ([0, 1, 2, 3, -1, 4], [1, 1, 1, 3, 7, 1]),    # one ends, and one starts in its place
        ([5, 4, 3, 2, 1, 0], [page, 1, 1, 1, 1, 1]),
    ]
    for parents, counts in steps:
        table, lengths, missing = ea.cache_update(cache, table, lengths, ints(parents), ints(counts))
        assert missing.tolist() == [0] * len(parents)
        rows, positions = new_tokens(lengths.tolist(), counts)
        k, v = (torch.randn(layers, rows.shape[0], hk, d, generator=g).to(dtype) for _ in range(2))
        hand.step(parents, counts, k, v)
        q = torch.randn(len(parents), hq, d, generator=g).to(dtype)
        for layer in range(layers):
            ea.cache_append(cache[layer], k[layer].cuda(), v[layer].cuda(), rows, positions, table)
            o = ea.paged_decode(q.cuda(), cache[layer], table, lengths)
            hand.check(cache, table, lengths, q, o, layer)
    before = table.clone()
    table, used = ea.cache_compact(cache, table, lengths)
    assert used.item() == len({p for row in before.tolist() for p in row if p >= 0}) == table.max().item() + 1
    for layer in range(layers):
        hand.check(cache, table, lengths, q, ea.paged_decode(q.cuda(), cache[layer], table, lengths), layer)


def test_chunks_of_a_prompt():
    """A prompt in two chunks: the second attends to the first's cached rows and its own."""
    hq, hk, d, n, page = 4, 2, 64, 90, 16
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(n, h, d, generator=g).to(BF) for h in (hq, hk, hk))
    cache = ea.paged_cache(10, page, hk, d)
    table, lengths, _ = ea.cache_update(cache, torch.zeros(1, 8, dtype=I32, device="cuda"), ints([0]), ints([-1]), ints([n]))
    rows, positions = new_tokens(lengths.tolist(), [n])
    first = 50
    ea.cache_append(cache, k[:first].cuda(), v[:first].cuda(), rows[:first], positions[:first], table)
    ea.cache_append(cache, k[first:].cuda(), v[first:].cuda(), rows[first:], positions[first:], table)
    keys, values = ea.cache_read(cache, rows, positions, table)
    plan = ea.packed_plan(ints([0, n]), n)
    o, _ = ea.packed_forward(q.cuda(), keys, values, plan, need_bwd=False)
    held = [pu.unpack(*pu.pack(t)) for t in (k, v)]
    want = packed64(q, held[0].float(), held[1].float(), [0, n], 1.5, d ** -0.5, True)[0]
    # Scores: 64 products added up in fp32, each step within 2^-24 of the sum of magnitudes, x
    # off by e; tau by e at most, sum |dp| <= 2 e gamma sum z <= 4 e sqrt(n).  The solver leaves
    # sum p off by 1e-5, and p is two bf16 terms, within 2^-16 of it.
    worst = (q.double().abs()[:, :2] * k.double().abs().amax(0)).sum(-1).max().item()
    e = 0.5 * d ** -0.5 * 64 * 2.0 ** -24 * worst
    check("chunks", o, want, (4 * e * n ** 0.5 + 1e-5 + 2.0 ** -16) * held[1].abs().max().item())
    last = ea.paged_decode(q[n - 1:].cuda(), cache, table, lengths)
    want, off = pu.paged64(q[n - 1:], pu.values(cache), table.cpu(), lengths.cpu(), None, page, 1.5, d ** -0.5)
    check("last", last, want, 0.0, off)


def test_a_step_in_a_graph():
    """A step captured once and replayed: tables, appended rows and attention as eager calls give
    them, with the program's own work between the replays.  Two graphs share the workspaces."""
    layers, hk, hq, d, page, width, pages, B = 2, 2, 4, 128, 16, 8, 40, 4
    cache = ea.paged_cache(pages, page, hk, d, layers)
    table, lengths = torch.full((B, width), -1, dtype=I32, device="cuda"), ints([0] * B)
    parents, counts = ints(range(B)), ints([1] * B)
    k, v = (torch.zeros(layers, B, hk, d, dtype=BF, device="cuda") for _ in range(2))
    q = torch.zeros(B, hq, d, dtype=BF, device="cuda")
    new = [torch.empty_like(table), torch.empty_like(lengths), torch.empty_like(lengths)]
    rows, positions = ints(range(B)), ints([0] * B)
    o = torch.zeros(layers, B, hq, d, dtype=BF, device="cuda")
    ws = [torch.empty(ea.cache_workspace(cache, B), dtype=torch.uint8, device="cuda"),
          torch.empty(ea.paged_decode_workspace(q, cache[0], table), dtype=torch.uint8, device="cuda")]

    def step():
        ea.cache_update(cache, table, lengths, parents, counts, *new, workspace=ws[0])
        table.copy_(new[0])
        lengths.copy_(new[1])
        torch.sub(lengths, 1, out=positions)
        for layer in range(layers):
            ea.cache_append(cache[layer], k[layer], v[layer], rows, positions, table)

    def attend():
        for layer in range(layers):
            ea.paged_decode(q, cache[layer], table, lengths, out=o[layer], workspace=ws[1])

    side = torch.cuda.Stream()
    state = [t.clone() for t in (cache, table, lengths)]
    with torch.cuda.stream(side):
        step()
        attend()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph, work in zip(graphs, (step, attend)):
        with torch.cuda.graph(graph):
            work()
    g = torch.Generator().manual_seed(1)
    for t, s in zip((cache, table, lengths), state):
        t.copy_(s)
    other = [t.clone() for t in state]  # the same by eager calls
    for n in range(40):
        p = list(range(B))
        if n % 7 == 3:
            p = [0, 0, 2, 1]
        if n == 20:
            p = [0, 1, -1, 3]
        parents.copy_(ints(p))
        for t in (k, v, q):
            t.copy_(torch.randn(t.shape, generator=g).to(BF))
        graphs[0].replay()
        graphs[1].replay()
        c2, t2, l2 = other
        t2, l2, missing = ea.cache_update(c2, t2, l2, parents, counts)
        eager = []
        for layer in range(layers):
            ea.cache_append(c2[layer], k[layer], v[layer], rows, l2 - 1, t2)
            eager.append(ea.paged_decode(q, c2[layer], t2, l2))
        other = [c2, t2, l2]
        assert torch.equal(table, t2) and torch.equal(lengths, l2) and torch.equal(new[2], missing)
        assert missing.tolist() == [0] * B
        assert torch.equal(cache, c2)
        for layer in range(layers):
            assert torch.equal(o[layer], eager[layer])
        if n % 10 == 9:
            torch.cuda.synchronize()
    vals = pu.values(cache[1])
    want, off = pu.paged64(q.cpu(), vals, table.cpu(), lengths.cpu(), None, page, 1.5, d ** -0.5)
    check("graph", o[1], want, 0.0, off)
