"""A chunk of a prompt with its own queries alone: they attend to the context in the pages and to
their own tokens before them."""
import pytest

torch = pytest.importorskip("torch")
from tests import pages_util as pu  # noqa: E402
from tests.layer_util import check, packed64  # noqa: E402

pytestmark = pytest.mark.gpu
I32, BF, F32 = torch.int32, torch.bfloat16, torch.float32


def ints(v):
    return torch.tensor(v, dtype=I32, device="cuda")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prompts,chunk,page,hq,hk,d", [([90], 40, 16, 4, 2, 64), ([300, 17, 129], 64, 32, 8, 2, 128), ([2100, 33], 100, 64, 2, 1, 64)])
def test_queries_of_a_chunk(prompts, chunk, page, hq, hk, d, dtype):
    import paper_2502_12082_amd as ea
    g = torch.Generator().manual_seed(chunk)
    # each prompt as chunks; the last chunk of each, at most `chunk` tokens, is asked for
    first = [(n - 1) // chunk * chunk for n in prompts]
    cache = ea.paged_cache(sum(-(-n // page) for n in prompts), page, hk, d)
    q, k, v = ([torch.randn(n, h, d, generator=g).to(dtype) for n in prompts] for h in (hq, hk, hk))
    width = -(-max(prompts) // page)
    table, lengths = torch.full((len(prompts), width), -1, dtype=I32, device="cuda"), ints([0] * len(prompts))
    at = [0] * len(prompts)
    while at != prompts:
        counts = [min(chunk, n - a) for n, a in zip(prompts, at)]
        table, lengths, missing = ea.cache_update(cache, table, lengths, ints(range(len(prompts))), ints(counts))
        assert missing.tolist() == [0] * len(prompts)
        places = [(r, a + i) for r, (a, c) in enumerate(zip(at, counts)) for i in range(c)]
        rows, positions = (ints(x) for x in zip(*places))
        new = [torch.cat([t[r][a:a + c] for r, (a, c) in enumerate(zip(at, counts))]).cuda() for t in (k, v)]
        ea.cache_append(cache, *new, rows, positions, table)
        at = [a + c for a, c in zip(at, counts)]
    places = [(r, a) for r, n in enumerate(prompts) for a in range(first[r], n)]
    rows, own_lengths = [r for r, _ in places], [a + 1 for _, a in places]
    queries = torch.stack([q[r][a] for r, a in places])
    o = ea.paged_decode(queries.cuda(), cache, table, ints(own_lengths), rows=ints(rows))
    want = torch.cat([packed64(q[r], *[pu.unpack(*pu.pack(t[r])).float() for t in (k, v)], [0, n], 1.5, d ** -0.5, True)[0][first[r]:]
                      for r, n in enumerate(prompts)])
    # how far a result may be off, of the definition over the pages
    same, off = pu.paged64(queries, pu.values(cache), table.cpu(), torch.tensor(own_lengths), rows, page, 1.5, d ** -0.5)
    assert (same - want).abs().max() < 1e-9
    check("chunk", o, want, 0.0, off)
