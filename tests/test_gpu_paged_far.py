"""Decoding over a cache in pages and in 4 bits, scores far from 0: what is left of a row are the
keys with the largest score, alike, however large it is."""
import pytest

torch = pytest.importorskip("torch")
from tests import pages_util as pu  # noqa: E402
from tests.layer_util import check, entmax64  # noqa: E402

pytestmark = pytest.mark.gpu
ea = None
I32, BF, F32 = torch.int32, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    global ea
    import paper_2502_12082_amd
    ea = paper_2502_12082_amd


def rows_of_ties(lengths, ties, page, hk, d, seed, largest=4.0, others=(0.5, 1.0, 1.5, 2.0, 3.0)):
    """(cache, table, which keys have the largest score): of row r's keys ties[r] have `largest`
    in dimension 0, the rest one of `others`, and all have 0 elsewhere; random values."""
    table, pages = pu.shuffled_table(lengths, page, 2, seed)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(pages, hk, 2, page // 16, 16, d, generator=g)
    x[:, :, 0] = 0.0
    top = []
    for r, n in enumerate(lengths):
        at = torch.arange(n)
        pages_of, tile, row = table[r].long()[at // page], at % page // 16, at % 16
        first = torch.randperm(n, generator=g)[:ties[r]]
        k = torch.tensor(others)[torch.randint(0, len(others), (n,), generator=g)]
        k[first] = largest
        for h in range(hk):
            x[pages_of, h, 0, tile, row, 0] = k
        top.append(first)
    code, scale = pu.pack(x)
    packed = torch.cat([(code[..., 0::2] + 16 * code[..., 1::2]).flatten(-2), scale.flatten(-2)], -1)
    return packed.to(torch.uint8), table, top


def compare(name, got, cache, table, lengths, top, page, alpha, rows=None):
    """p = 1 / t for t ties.  The solver leaves the sum of p off by 1e-6; every p and each step of
    their sums is a rounding or two, and a general power 2^-18."""
    vals = pu.values(cache)
    hq, hk = got.shape[1], vals.shape[2]
    want = torch.zeros(got.shape, dtype=torch.float64)
    off = torch.zeros(got.shape, dtype=torch.float64)
    for i in range(got.shape[0]):
        r = i if rows is None else rows[i]
        _, v, there = pu.keys_of(vals, table, r, lengths[r], page)
        assert there.all()
        t = len(top[r])
        assert t and torch.allclose(entmax64(torch.zeros(1, t, dtype=torch.float64), alpha)[0], torch.full((1, t), 1 / t, dtype=torch.float64))
        v = v[top[r]].repeat_interleave(hq // hk, 1)
        want[i] = v.mean(0)
        off[i] = v.abs().mean(0) * (1e-6 + (t + 16) * 2.0 ** -24 + (0 if alpha in (1.25, 1.5, 2.0) else 2.0 ** -18))
    check(name, got, want, 0.0, off)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("alpha", [1.5, 2.0, 1.25, 1.4])
@pytest.mark.parametrize("power", [4, 10, 18, 22, 23, 24, 25, 40, 100])
def test_largest_scores(power, alpha, dtype, wide):
    """x of 2^power and its neighbours, and below them; one key, two, three, hundreds with the largest."""
    lengths, ties, page, hk, d = [900, 37, 1300, 1, 600, 250], [1, 2, 1300, 1, 3, 200], 16, 2, 64
    cache, table, top = rows_of_ties(lengths, ties, page, hk, d, power)
    if wide:
        table = torch.cat([table, torch.full((len(lengths), 130), -1, dtype=I32)], 1)
    # x = (alpha - 1) scale q k: 4 in dimension 0 is (about, where alpha is 1.4) 2^power times 1, 1.5, 1.25, 1.75
    q = torch.zeros(len(lengths), 4, d)
    q[:, :, 0] = 2.0 ** (power - 2) * torch.tensor([1.0, 1.5, 1.25, 1.75])
    got = ea.paged_decode(q.to(dtype).cuda(), cache.cuda(), table.cuda(), torch.tensor(lengths, dtype=I32).cuda(), alpha=alpha,
                          scale=1.0 / (alpha - 1.0))
    compare("far", got, cache, table, lengths, top, page, alpha)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("power", [10, 24, 30])
def test_largest_scores_below_zero(power, wide):
    """All scores far below 0."""
    lengths, ties, page = [700, 40], [2, 1], 32
    cache, table, top = rows_of_ties(lengths, ties, page, 1, 64, power, -0.5, (-1.0, -1.5, -2.0, -4.0))
    if wide:
        table = torch.cat([table, torch.full((2, 65), -1, dtype=I32)], 1)
    q = torch.zeros(2, 2, 64, dtype=BF)
    q[:, :, 0] = 2.0 ** power
    got = ea.paged_decode(q.cuda(), cache.cuda(), table.cuda(), torch.tensor(lengths, dtype=I32).cuda(), alpha=1.5, scale=2.0)
    compare("below", got, cache, table, lengths, top, page, 1.5)


@pytest.mark.parametrize("copies,n", [(1, 20000), (80, 5000)])
@pytest.mark.parametrize("power", [18, 24, 60])
def test_dense_ties(power, copies, n):
    """More keys with the largest score than a workgroup's threads keep: (1) sixteen waves, (80) four."""
    lengths, ties, page, alpha = [n, 300], [n - 7, 2], 64, 1.5
    cache, table, top = rows_of_ties(lengths, ties, page, 1, 64, power)
    q = torch.zeros(2 * copies, 2, 64, dtype=BF)
    q[:, :, 0] = 2.0 ** (power - 2)
    rows = [0, 1] * copies
    lengths_of = torch.tensor([lengths[r] for r in rows], dtype=I32)
    got = ea.paged_decode(q.cuda(), cache.cuda(), table.cuda(), lengths_of.cuda(), rows=torch.tensor(rows, dtype=I32).cuda(),
                          alpha=alpha, scale=2.0)
    compare("dense", got[:2], cache, table, lengths, top, page, alpha, rows=[0, 1])
    assert torch.equal(got[:2].repeat(copies, 1, 1), got)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("power", [20, 100, 106, 112, 118, 122, 123])
def test_small_queries(power, dtype, wide):
    """Queries next to the smallest numbers enter the scores within 2^-124, or 2^-19 (fp32: 2^-29) of
    their largest value: two keys, alpha 2, p of the first is (1 + x_0 - x_1) / 2."""
    table = torch.zeros(1, 200 if wide else 1, dtype=I32)
    x = torch.zeros(1, 1, 2, 1, 16, 64)
    x[0, 0, 0, 0, :2, 0] = torch.tensor([4.0, 3.0])
    x[0, 0, 1, 0, 0, 0] = 1.0
    code, scale = pu.pack(x)
    cache = torch.cat([(code[..., 0::2] + 16 * code[..., 1::2]).flatten(-2), scale.flatten(-2)], -1).to(torch.uint8)
    q = torch.zeros(1, 1, 64, dtype=torch.float64)
    q[..., 0] = (1 + 37 / 128) * 2.0 ** -power
    c = 2.0 ** (power - 2)
    got = ea.paged_decode(q.to(dtype).cuda(), cache.cuda(), table.cuda(), torch.tensor([2], dtype=I32).cuda(), alpha=2.0, scale=c)
    want = torch.zeros(1, 1, 64, dtype=torch.float64)
    want[..., 0] = 0.5 * (1 + c * float(q[0, 0, 0]))
    # (x of up to 1.3 is a product in fp32; the solver's sum is off by 1e-6)
    off = 0.5 * c * 7 * max(2.0 ** -124, float(q[0, 0, 0]) * 2.0 ** (-29 if dtype == F32 else -19)) + 1e-6 + 8 * 2.0 ** -24
    check("small", got, want, 0.0, torch.where(want > 0, off, 0.0))
