"""prefix_decode: fp32 keys at the edge of the support, strides of a prefix that is
not there, waves of several runs, scores that are not finite."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import check, decode64  # noqa: E402
from test_gpu_decode import ATOL, compare, ea, make, run  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("alpha", [1.25, 1.7, 2.5, 3.0])
@pytest.mark.parametrize("c", [0.03, 0.4, 1.0, 6.0])
def test_fp32_exponents(ea, alpha, c):
    """fp32 with every kind of exponent; all keys, many and few in the support."""
    x = make([2500, 9, 40], 1100, 2500, 4, 2, 64, F32, c=c, seed=31)
    compare(run(ea, x, alpha, max_iter=60), x, alpha, "c%g a%g" % (c, alpha), c)


def edge_keys(x, alpha, scale):
    """Puts every request's last own key at the threshold that the other keys have."""
    a, s = (float(torch.tensor(t, dtype=torch.float32)) for t in (alpha, scale))
    gamma = 1.0 / (a - 1.0)
    B, hq, d = x["q"].shape
    for b in range(B):
        n = int(x["lengths"][b])
        for h in range(hq):
            q = x["q"][b, h].double().cpu()
            keys = x["k"][b, :n - 1, h].double().cpu()
            if x["pk"] is not None:
                keys = torch.cat([x["pk"][:, h].double().cpu(), keys])
            y = (a - 1.0) * s * (keys @ q)
            top = float(y.max())
            lo, hi = top - 1.0, top
            for _ in range(80):
                mid = 0.5 * (lo + hi)
                lo, hi = (mid, hi) if float(((y - mid).clamp_min(0.0) ** gamma).sum()) >= 1.0 else (lo, mid)
            x["k"][b, n - 1, h] = (q * (lo / ((a - 1.0) * s * float(q @ q)))).float().cuda()


@pytest.mark.parametrize("alpha", [2.5, 3.0])
@pytest.mark.parametrize("c,prefix,own", [(20.0, 0, 40), (6.0, 300, 200), (0.3, 1000, 1500), (0.05, 1000, 1500)])
@pytest.mark.parametrize("d", [64, 128])
def test_fp32_keys_at_the_edge(ea, alpha, c, prefix, own, d):
    """alpha > 2: p = z^gamma has no bounded slope at z = 0, so that a score off
    by 1e-6 has p off by 1e-3 at alpha 3.  Scores near the edge are exact, as in
    attention: 5e-5 as everywhere (scores off by 2^-24 sqrt(d) |x| times the
    slope gamma z^(gamma - 1) beyond the edge's neighbourhood z > 0.01 max(1,
    |tau|): 0.5 (0.2)^-0.5 4e-6 at |x| = 20, 0.5 (0.01)^-0.5 3e-7 at |x| < 1; p
    in 24 bits)."""
    x = make([own, own - 7, own // 2, 3], prefix, own, 4, 4, d, F32, c=c, seed=32)
    edge_keys(x, alpha, d ** -0.5)
    want = decode64(x["q"], x["k"], x["v"], x["lengths"].tolist(), x["pk"], x["pv"], alpha, d ** -0.5)
    check("a%g c%g" % (alpha, c), run(ea, x, alpha, max_iter=64), want, 5e-5)


def test_fp32_keys_at_the_edge_of_many_rows(ea):
    """The same with a wave to every row (512 rows and more)."""
    g = torch.Generator().manual_seed(33)
    lengths = torch.randint(2, 40, (130,), generator=g).tolist()
    x = make(lengths, 0, 40, 4, 4, 64, F32, c=20.0, seed=34)
    edge_keys(x, 3.0, 0.125)
    want = decode64(x["q"], x["k"], x["v"], lengths, None, None, 3.0, 0.125)
    check("many", run(ea, x, 3.0, max_iter=64), want, 5e-5)


def test_no_prefix_takes_no_strides(ea):
    """Without a prefix a query's strides stand for nothing but the query's."""
    x = make([9, 5], 0, 9, 2, 1, 64, BF, seed=36)
    want = run(ea, x)
    far = torch.empty(2, (1 << 24) + 64, dtype=BF, device="cuda")
    q = far[:, :128].view(2, 2, 64)
    q.copy_(x["q"])
    assert torch.equal(run(ea, dict(x, q=q)), want)


@pytest.mark.parametrize("prefix,requests,d,dtype", [(33001, 20, 64, BF), (100001, 20, 64, BF), (33001, 12, 128, F32)])
def test_several_runs_to_a_wave(ea, prefix, requests, d, dtype):
    """Prefixes whose waves take 2 (33001) and 6 runs, the last ones fewer, of
    two row tiles; some rows of the first, middle and last request and key head."""
    x = make([b % 5 for b in range(requests)], prefix, 5, 32, 8, d, dtype, seed=35)
    got = run(ea, x)
    for b, h in ((0, 0), (0, 31), (requests // 2, 13), (requests - 1, 5), (requests - 1, 31)):
        one = lambda t, dim: t.narrow(dim, h // 4, 1)
        want = decode64(x["q"][b:b + 1, h:h + 1], one(x["k"], 2)[b:b + 1], one(x["v"], 2)[b:b + 1],
                        x["lengths"][b:b + 1].tolist(), one(x["pk"], 1), one(x["pv"], 1), 1.5, d ** -0.5)
        check("%d %d" % (b, h), got[b:b + 1, h:h + 1], want, ATOL[dtype])


@pytest.mark.parametrize("prefix,own", [(0, 30), (200, 700), (5000, 10)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype,alpha", [(BF, 1.5), (BF, 2.5), (F32, 3.0)])
def test_scores_that_are_not_finite(ea, prefix, own, bad, dtype, alpha):
    """A query that is not finite, in one element (scores of +-inf, or NaN) or in
    all (NaN): its row of O is 0, as in attention, and the others are unchanged."""
    x = make([own, own - 3], prefix, own, 4, 2, 64, dtype, seed=37)
    want = run(ea, x, alpha, max_iter=40)
    x["q"] = x["q"].clone()
    x["q"][1, 2] = bad
    x["q"][0, 1, 5] = bad
    got = run(ea, x, alpha, max_iter=40)
    assert not got[1, 2].any() and not got[0, 1].any()
    got[1, 2], got[0, 1] = want[1, 2], want[0, 1]
    assert torch.equal(got, want)
