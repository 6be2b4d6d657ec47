"""Decoding over a cache in pages and in 4 bits on the GPU."""
import pytest

torch = pytest.importorskip("torch")
from tests import pages_util as pu  # noqa: E402
from tests.layer_util import check  # noqa: E402

pytestmark = pytest.mark.gpu
ea = None
I32, BF, F32 = torch.int32, torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def library():
    global ea
    import paper_2502_12082_amd
    ea = paper_2502_12082_amd


def queries(n, hq, d, dtype, c, seed):
    return (torch.randn(n, hq, d, generator=torch.Generator().manual_seed(seed)) * c).to(dtype)


def widened(table, page, wide):
    """The table as it is (short rows: one launch), or with room for more tokens than a workgroup holds."""
    more = -(-2064 // page) if wide else 0
    return torch.cat([table, torch.full((table.shape[0], more), -1, dtype=I32)], 1)


def compare(name, q, cache, table, lengths, rows=None, alpha=1.5, scale=None, **kw):
    page = 16 * cache.shape[3]
    scale_ = q.shape[-1] ** -0.5 if scale is None else scale
    got = ea.paged_decode(q.cuda(), cache.cuda(), table.cuda(), lengths.cuda(), rows=None if rows is None else rows.cuda(),
                          alpha=alpha, scale=scale, **kw)
    want, off = pu.paged64(q, pu.values(cache), table, lengths, rows, page, alpha, scale_)
    assert got.shape == q.shape and got.dtype == q.dtype
    check(name, got, want, 0.0, off)
    return got


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("alpha", [1.5, 1.25, 2.0, 1.4])
@pytest.mark.parametrize("hq,hk,d,page,lengths", [
    (1, 1, 64, 16, [1, 0, 17]), (4, 4, 128, 32, [5, 33, 300]), (8, 2, 128, 16, [64, 1500, 3]), (14, 2, 64, 64, [129, 63, 1024]),
    (12, 1, 128, 128, [1025, 1023]), (40, 2, 64, 16, [700, 31]), (9, 3, 128, 1024, [2100, 1])])
def test_decode(hq, hk, d, page, lengths, alpha, dtype, wide):
    seed = hq * 100 + page
    table, pages = pu.shuffled_table(lengths, page, 2, seed, width=max(-(-max(lengths) // page) + 1, 2))
    table = widened(table, page, wide)
    cache = pu.filled(torch.empty(pages, hk, 2, page // 16, 17 * d // 2, dtype=torch.uint8), seed)
    c = {1.5: 1.0, 1.25: 2.0, 2.0: 0.7, 1.4: 4.0}[alpha]
    q = queries(len(lengths), hq, d, dtype, c, seed)
    compare("decode", q, cache, table, torch.tensor(lengths, dtype=I32), alpha=alpha)


@pytest.mark.parametrize("c,alpha", [(0.05, 1.5), (0.3, 1.25), (8.0, 1.5), (0.0, 2.0), (0.2, 1.1)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_dense_and_sparse_rows(c, alpha, dtype):
    """Rows whose probabilities are nearly all positive (more than a wave's lists hold, and than a workgroup's), or few."""
    lengths = [3000, 400, 5000]
    table, pages = pu.shuffled_table(lengths, 64, 0, 3)
    cache = pu.filled(torch.empty(pages, 2, 2, 4, 1088, dtype=torch.uint8), 5)
    compare("dense", queries(3, 6, 128, dtype, c, 1), cache, table, torch.tensor(lengths, dtype=I32), alpha=alpha)


@pytest.mark.parametrize("wide", [False, True])
def test_rows_and_lengths(wide):
    """Several queries to a row, rows in any order, lengths past both ends, rows that there are not."""
    table, pages = pu.shuffled_table([200, 90, 40], 16, 4, 9)
    cache = pu.filled(torch.empty(pages, 2, 2, 1, 544, dtype=torch.uint8), 7)
    rows = torch.tensor([1, 0, 0, 0, 2, -1, 3, 2 ** 31 - 1, -2 ** 31, 1], dtype=I32)
    lengths = torch.tensor([90, 198, 199, 200, 0, 50, 50, 50, 50, -3], dtype=I32)
    q = queries(10, 4, 64, BF, 1.0, 2)
    got = compare("rows", q, cache, widened(table, 16, wide), lengths, rows)
    assert (got[4:].float() == 0).all()
    # lengths behind the table's width, and max_length
    many = torch.tensor([2 ** 31 - 1, 1000, 208], dtype=I32)
    table[1, 6:] = table[0, 6:]
    table[2, 3:] = table[0, 3:]
    table = widened(table, 16, wide)
    full = compare("width", q[:3], cache, table, many)
    cut = ea.paged_decode(q[:3].cuda(), cache.cuda(), table.cuda(), many.cuda(), max_length=100)
    want, off = pu.paged64(q[:3], pu.values(cache), table, many.clamp_max(100), None, 16, 1.5, 64 ** -0.5)
    check("max_length", cut, want, 0.0, off)
    assert not torch.equal(full, cut)
    none = ea.paged_decode(q[:3].cuda(), cache.cuda(), table.cuda(), many.cuda(), max_length=0)
    assert (none == 0).all()
    assert ea.paged_decode(q[:0].cuda(), cache.cuda(), table.cuda(), many[:0].cuda()).shape == (0, 4, 64)


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_there_are_not(dtype, wide):
    """Entries of no page have no keys: in the middle, at the end, all of them."""
    table, pages = pu.shuffled_table([300, 300, 1400], 16, 2, 4)
    table = widened(table, 16, wide)
    cache = pu.filled(torch.empty(pages, 1, 2, 1, 1088, dtype=torch.uint8), 8)
    table[0, 3:7] = torch.tensor([-1, pages, 2 ** 31 - 1, -2 ** 31], dtype=I32)
    table[1] = -1
    table[2, 64:] = pages
    lengths = torch.tensor([300, 300, 1400], dtype=I32)
    got = compare("holes", queries(3, 2, 128, dtype, 1.0, 3), cache, table, lengths)
    assert (got[1] == 0).all()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_not_finite(dtype, wide):
    """NaN keys have no probability; NaN values reach what they are used in; queries that
    are not finite give 0; bytes behind a row's end and in pages of others say nothing."""
    lengths = [100, 100, 100, 100, 100]
    table, pages = pu.shuffled_table(lengths, 32, 2, 6)
    table = widened(table, 32, wide)
    cache = pu.filled(torch.empty(pages, 2, 2, 2, 1088, dtype=torch.uint8), 9)
    for r in range(5):
        last = cache[int(table[r, 3])]
        for at in range(4, 32):  # tokens 100 ..: NaN scales
            last[:, :, at // 16, 1024 + at % 16 * 4:1024 + at % 16 * 4 + 4] = 255
    q = queries(5, 4, 128, dtype, 1.0, 4)
    key = lambda r, at, head, which: cache[int(table[r, at // 32]), head, which, at % 32 // 16]
    for at in (0, 50, 99):
        key(0, at, 0, 0)[1024 + at % 16 * 4 + 2] = 255  # one block of row 0's keys, head 0
    q[1, 0, 5], q[1, 1, 70], q[1, 3, 127] = float("nan"), float("inf"), float("-inf")
    q[2] = 0  # every key the same: all have a probability
    lengths = torch.tensor(lengths, dtype=I32)
    got = compare("nan", torch.where(torch.isfinite(q), q, 0.0), cache, table, lengths)
    bad = ea.paged_decode(q.cuda(), cache.cuda(), table.cuda(), lengths.cuda()).cpu()
    assert (bad[1, [0, 1, 3]] == 0).all()
    assert torch.equal(bad[1, 2], got[1, 2].cpu()) and torch.equal(bad[[0, 2, 3, 4]], got[[0, 2, 3, 4]].cpu())
    # a NaN value: of row 2 (all keys used) in dims 32 .. 63 of head 1
    key(2, 64, 1, 1)[1024 + 0 * 4 + 1] = 255
    nan = ea.paged_decode(q.cuda(), cache.cuda(), table.cuda(), lengths.cuda()).cpu()
    assert torch.isnan(nan[2, 2:, 32:64]).all() and not torch.isnan(nan[2, :2]).any()
    assert not torch.isnan(nan[2, 2:, :32]).any() and not torch.isnan(nan[2, 2:, 64:]).any()
    assert not torch.isnan(nan[[0, 1, 3, 4]]).any()


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_magnitudes(dtype, wide):
    """Queries and keys whose blocks differ by many powers of two."""
    lengths = [260, 100]
    table, pages = pu.shuffled_table(lengths, 16, 0, 5)
    table = widened(table, 16, wide)
    cache = pu.filled(torch.empty(pages, 1, 2, 1, 1088, dtype=torch.uint8), 11)
    scales = cache[..., 1024:].view(pages, 1, 2, 1, 16, 4)
    scales[:, :, 0] += torch.tensor([20, 0, 246, 3], dtype=torch.uint8)  # (246: less 10)
    q = queries(2, 4, 128, F32, 1.0, 6)
    q[:, :, :32] *= 2.0 ** -20
    q[:, :, 64:96] *= 2.0 ** 10
    q[:, 1, 3] = 100.0
    q[:, 2, 40] = 0.0
    q[:, 3, 96:] *= 2.0 ** -100
    compare("magnitudes", q.to(dtype), cache, table, torch.tensor(lengths, dtype=I32), scale=0.02)


@pytest.mark.parametrize("wide", [False, True])
def test_strides_out_and_workspace(wide):
    table, pages = pu.shuffled_table([500, 70], 32, 1, 12)
    table = widened(table, 32, wide)
    cache = pu.filled(torch.empty(pages, 2, 2, 2, 1088, dtype=torch.uint8), 13)
    lengths = torch.tensor([500, 70], dtype=I32)
    q = queries(2, 8, 128, BF, 1.0, 7)
    want = compare("plain", q, cache, table, lengths)
    rows = torch.zeros(2, 3, 8, 128, dtype=BF, device="cuda")
    rows[:, 1] = q.cuda()
    out = torch.full((2, 8, 256), 5.0, dtype=BF, device="cuda")
    around = torch.full((2, table.shape[1] + 4), -1, dtype=I32, device="cuda")
    around[:, 2:2 + table.shape[1]] = table.cuda()
    t = around[:, 2:2 + table.shape[1]]
    ws = torch.full((ea.paged_decode_workspace(q, cache, t),), 0xFF, dtype=torch.uint8, device="cuda")
    for byte in (0xFF, 0x7F, 0):
        ws.fill_(byte)
        got = ea.paged_decode(rows[:, 1], cache.cuda(), t, lengths.cuda(), out=out[..., 128:], workspace=ws)
        assert got.data_ptr() == out[..., 128:].data_ptr()
        assert torch.equal(got, want) and (out[..., :128] == 5).all()


def test_long_row():
    """The longest rows, and a pool of more than 2^32 bytes."""
    page, n = 1024, 131072
    pages = (5 << 30) // (page * 2 * 136) if torch.cuda.get_device_properties(0).total_memory > 1 << 36 else 200
    table = torch.full((2, 128), -1, dtype=I32)
    table[0] = torch.arange(pages - 128, pages)
    table[1] = torch.arange(128, 0, -1)
    some = pu.filled(torch.empty(256, 2, 2, 64, 1088, dtype=torch.uint8), 17)
    cache = torch.zeros(pages, 2, 2, 64, 1088, dtype=torch.uint8, device="cuda")
    cache[pages - 128:], cache[1:129] = some[:128].cuda(), some[128:].cuda()
    lengths = torch.tensor([n, n - 777], dtype=I32)
    q = queries(2, 2, 128, BF, 1.0, 8)
    got = ea.paged_decode(q.cuda(), cache, table.cuda(), lengths.cuda())
    near = torch.stack([torch.arange(128), 128 + torch.arange(127, -1, -1)]).int()
    vals = pu.values(some)
    want, off = pu.paged64(q, vals, near, lengths, None, page, 1.5, 128 ** -0.5)
    check("long", got, want, 0.0, off)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hk,lengths", [(3, 1, [2000, 1500, 64]), (8, 1, [2040, 700]), (24, 2, [1024, 1000]),
                                           (16, 1, [1024, 900, 15]), (40, 2, [1024, 777])])
@pytest.mark.parametrize("c,alpha", [(0.02, 1.5), (0.3, 1.25), (0.5, 1.15)])
def test_dense_short_rows(hq, hk, lengths, c, alpha, dtype):
    """Short rows with more scores above the bound than one workgroup's lists hold."""
    table, pages = pu.shuffled_table(lengths, 16, 0, hq)
    cache = pu.filled(torch.empty(pages, hk, 2, 1, 544, dtype=torch.uint8), hq)
    compare("short", queries(len(lengths), hq, 64, dtype, c, hq), cache, table, torch.tensor(lengths, dtype=I32), alpha=alpha)


@pytest.mark.parametrize("copies,n,c,alpha", [
    (1, 20000, 0.05, 1.25),    # more entries than a large workgroup's threads keep
    (60, 20000, 0.05, 1.25), (60, 6000, 0.3, 1.5),  # (300 rows) and than a small one's
    (220, 5000, 1.0, 1.5), (220, 5000, 0.05, 1.5)])  # (1100 rows) first waves alone, and all of them
def test_many_queries_of_few_rows(copies, n, c, alpha):
    """Five queries, again and again: as many rows as choose each of the kernels' forms."""
    lengths = torch.tensor([n, n - 1, n // 2, 33, 0], dtype=I32)
    table, pages = pu.shuffled_table([n, n // 2 + 1], 64, 1, 3)
    cache = pu.filled(torch.empty(pages, 1, 2, 4, 544, dtype=torch.uint8), 21)
    rows = torch.tensor([0, 0, 1, 1, 0], dtype=I32)
    q = queries(5, 1, 64, BF, c, 9)
    want, off = pu.paged64(q, pu.values(cache), table, lengths, rows, 64, alpha, 64 ** -0.5)
    got = ea.paged_decode(q.repeat(copies, 1, 1).cuda(), cache.cuda(), table.cuda(), lengths.repeat(copies).cuda(),
                          rows=rows.repeat(copies).cuda(), alpha=alpha)
    check("many", got, want.repeat(copies, 1, 1), 0.0, off.repeat(copies, 1, 1))
    assert torch.equal(got[:5].repeat(copies, 1, 1), got)  # (whichever workgroup: the same)


def test_same_again_and_other_streams():
    """The same bits at every call, on any stream, and with calls on two streams at once."""
    table, pages = pu.shuffled_table([5000, 300, 2222], 32, 1, 12)
    cache = pu.filled(torch.empty(pages, 2, 2, 2, 1088, dtype=torch.uint8), 13).cuda()
    lengths = torch.tensor([5000, 300, 2222], dtype=I32).cuda()
    table = table.cuda()
    q = [queries(3, 6, 128, BF, c, 7).cuda() for c in (1.0, 0.1)]
    want = [ea.paged_decode(x, cache, table, lengths, alpha=a) for x in q for a in (1.5, 1.25)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for n, (x, a) in enumerate((x, a) for x in q for a in (1.5, 1.25)):
            with torch.cuda.stream(streams[n % 2]):
                got.append(ea.paged_decode(x, cache, table, lengths, alpha=a))
    torch.cuda.synchronize()
    for n, g in enumerate(got):
        assert torch.equal(g, want[n % 4])


@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("c,alpha,scale", [(100.0, 1.5, 0.1), (100.0, 2.0, 0.1), (1000.0, 1.25, 0.1), (1.0, 1.01, 0.1),
                                           (1.0, 1.9, 1e-4), (1.0, 1.5, 1e-30), (3.0, 1.001, 1.0)])
def test_steep_and_flat(c, alpha, scale, dtype, wide):
    """Scores of thousands, where one or two keys have it all, and all alike; alpha next to 1."""
    lengths = [900, 37]
    table, pages = pu.shuffled_table(lengths, 16, 0, 5)
    table = widened(table, 16, wide)
    cache = pu.filled(torch.empty(pages, 1, 2, 1, 544, dtype=torch.uint8), 31)
    compare("steep", queries(2, 3, 64, dtype, c, 8), cache, table, torch.tensor(lengths, dtype=I32), alpha=alpha,
            scale=scale, max_iter=64)


@pytest.mark.parametrize("wide", [False, True])
def test_iterations_and_limits(wide):
    """No iterations, none left out (tol 0), and products that overflow: finite, and 0 in the end."""
    lengths = torch.tensor([900, 37], dtype=I32)
    table, pages = pu.shuffled_table([900, 37], 16, 0, 5)
    table = widened(table, 16, wide).cuda()
    cache = pu.filled(torch.empty(pages, 1, 2, 1, 544, dtype=torch.uint8), 31).cuda()
    q = queries(2, 3, 64, F32, 1.0, 8).cuda()
    args = (cache, table, lengths.cuda())
    once = ea.paged_decode(q, *args, max_iter=0)
    all_of_them = ea.paged_decode(q, *args, max_iter=64, tol=0.0)
    assert torch.isfinite(once).all()
    want, off = pu.paged64(q.cpu(), pu.values(cache), table.cpu(), lengths, None, 16, 1.5, 64 ** -0.5)
    check("tol 0", all_of_them, want, 0.0, off)
    assert (ea.paged_decode(q * 1e30, *args, scale=1e30) == 0).all()  # (scores times scale past fp32)
    assert torch.isfinite(ea.paged_decode(q * 1e15, *args)).all()
