"""prefix_decode against the definition in 64 bits.

Tolerances beside the output's rounding: scores are off by 2^-24 sqrt(d) |x|
(1e-6 for these inputs, c times that for larger queries), p by twice that and
sum p by the solver's tolerance 1e-6, both times |v| <= 5 over the support."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import check, decode64, packed64, rotary64  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
ATOL = {BF: 2e-4, F32: 5e-5}


@pytest.fixture(scope="module", autouse=True)
def ea():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_12082_amd
    return paper_2502_12082_amd


def make(lengths, prefix, cap, hq, hk, d, dtype, c=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    B = len(lengths)
    r = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    x = {"q": (c * torch.randn(B, hq, d, generator=g)).to(dtype).cuda(), "k": r(B, cap, hk, d), "v": r(B, cap, hk, d),
         "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
         "pk": r(prefix, hk, d) if prefix else None, "pv": r(prefix, hk, d) if prefix else None}
    for b, n in enumerate(lengths):  # what lies behind a request's keys reaches nothing
        x["k"][b, max(n, 0):] = float("nan")
        x["v"][b, max(n, 0):] = float("nan")
    return x


def run(ea, x, alpha=1.5, **kw):
    return ea.prefix_decode(x["q"], x["k"], x["v"], x["lengths"], x["pk"], x["pv"], alpha=alpha, **kw)


def compare(got, x, alpha, label, c=1.0):
    d = x["q"].shape[-1]
    want = decode64(x["q"], x["k"], x["v"], x["lengths"].tolist(), x["pk"], x["pv"], alpha, d ** -0.5)
    check(label, got, want, ATOL[x["q"].dtype] * max(1.0, c))


@pytest.mark.parametrize("lengths,prefix,cap", [([1], 0, 1), ([0], 0, 5), ([0, 3], 1, 8), ([33, 0, 32, 64], 0, 64),
                                                ([5, 700, 128, 0, 129], 300, 700), ([0, 0], 65, 0), ([2] * 70, 129, 3)])
@pytest.mark.parametrize("hq,hk,d,dtype,alpha", [(4, 2, 64, BF, 1.5), (8, 1, 128, BF, 1.5), (7, 7, 128, BF, 1.25),
                                                 (4, 1, 64, F32, 1.5), (2, 2, 128, F32, 2.0), (6, 3, 64, BF, 1.7),
                                                 (40, 1, 64, BF, 1.5)])
def test_against_definition(ea, lengths, prefix, cap, hq, hk, d, dtype, alpha):
    x = make(lengths, prefix, cap, hq, hk, d, dtype, seed=prefix + hq)
    compare(run(ea, x, alpha), x, alpha, "%s p%d %d/%d d%d %s a%g" % (lengths[:5], prefix, hq, hk, d, dtype, alpha))


@pytest.mark.parametrize("c", [0.0, 0.03, 0.4, 20.0])
@pytest.mark.parametrize("alpha", [1.5, 1.25, 2.0, 2.5])
def test_supports(ea, c, alpha):
    """Every key in the support (more than are kept at once), many, and one."""
    x = make([4000, 9], 3100, 4000, 4, 2, 64, BF, c=c, seed=1)
    compare(run(ea, x, alpha, max_iter=40), x, alpha, "c%g a%g" % (c, alpha), c)


@pytest.mark.parametrize("c", [0.0, 0.3, 1.0, 8.0])
@pytest.mark.parametrize("d,dtype", [(128, BF), (64, F32)])
def test_many_rows(ea, c, d, dtype):
    """Rows enough for a wave each: every key in the support, many, few."""
    g = torch.Generator().manual_seed(10)
    lengths = torch.randint(0, 90, (40,), generator=g).tolist()
    x = make(lengths, 1500, 90, 16, 2, d, dtype, c=c, seed=11)
    compare(run(ea, x), x, 1.5, "c%g d%d" % (c, d), c)


def test_long_prefix(ea):
    x = make([100, 0, 50], 100000, 100, 4, 2, 128, BF, c=1.0, seed=2)
    compare(run(ea, x), x, 1.5, "long")


def test_lengths_outside(ea):
    """Lengths below 0 and above the capacity are taken as 0 and the capacity."""
    x = make([30, 0], 10, 30, 4, 2, 64, BF, seed=3)
    want = run(ea, x)
    x["lengths"].copy_(torch.tensor([1 << 30, -5], dtype=torch.int32))
    assert torch.equal(run(ea, x), want)


def test_far_rows(ea):
    """A cache whose offsets pass 32 bits, in elements and bytes."""
    B, cap, hk, d = 66, 65536, 8, 64
    g = torch.Generator().manual_seed(12)
    x = make([0] * B, 0, 1, 16, hk, d, BF, seed=12)
    x["k"], x["v"] = (torch.zeros(B, cap, hk, d, dtype=BF, device="cuda") for _ in range(2))
    x["lengths"][0], x["lengths"][B - 1] = 100, cap
    for b, n in ((0, 100), (B - 1, cap)):
        for name in ("k", "v"):
            x[name][b, :n] = torch.randn(n, hk, d, generator=g).to(BF).cuda()
    got = run(ea, x)
    last = {n: (t[B - 1:] if t is not None else None) for n, t in x.items()}
    first = {n: (t[:1] if t is not None else None) for n, t in x.items()}
    compare(got[B - 1:], last, 1.5, "last")
    compare(got[:1], first, 1.5, "first")
    assert not got[1:B - 1].any()


def test_no_requests(ea):
    x = make([], 5, 3, 2, 1, 64, BF)
    assert run(ea, x).shape == (0, 2, 64)


def test_parameters_in_tensors(ea):
    """A call takes what its parameters hold when it is made."""
    x = make([300, 41], 20, 4, 2, 1, 64, BF, c=2.0, seed=13)
    alpha, scale = torch.tensor(1.25), torch.tensor(0.1)
    for a, s in ((1.25, 0.1), (2.0, 0.3)):
        alpha.fill_(a), scale.fill_(s)
        got = run(ea, x, alpha, scale=scale)
        assert torch.equal(got, run(ea, x, float(alpha), scale=float(scale)))


def test_equal_scores(ea):
    """Ties: every key the same, so that each has probability 1 / n."""
    x = make([100, 40], 60, 100, 2, 1, 64, BF, seed=4)
    x["k"][:] = x["k"][0, 0, 0]
    x["pk"][:] = x["k"][0, 0, 0]
    compare(run(ea, x), x, 1.5, "ties")


def test_non_finite_values_of_zero_probability(ea):
    """A key whose score is out of reach may have any value; a key that is NaN has probability 0."""
    x = make([200, 100], 100, 200, 2, 1, 64, BF, c=2.0, seed=5)
    want = run(ea, x)
    x["k"] = torch.cat([x["k"], x["k"][:, :1]], 1)
    x["v"] = torch.cat([x["v"], x["v"][:, :1]], 1)
    x["k"][0, 200] = float("nan")
    x["v"][0, 200] = float("inf")
    x["lengths"][0] = 201
    assert torch.equal(run(ea, x), want)


def test_layouts(ea):
    """Head-major caches, a prefix inside a prompt's rows, a padded query."""
    x = make([90, 17], 70, 96, 4, 2, 64, BF, seed=6)
    want = run(ea, x)
    major = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)
    rows = torch.zeros(80, 2, 2 * 64, dtype=BF, device="cuda")
    rows[5:75, :, :64], rows[5:75, :, 64:] = x["pk"], x["pv"]
    q = torch.zeros(2, 4, 72, dtype=BF, device="cuda")
    q[..., :64] = x["q"]
    y = dict(x, k=major(x["k"]), v=major(x["v"]), pk=rows[5:75, :, :64], pv=rows[5:75, :, 64:], q=q[..., :64])
    out = torch.zeros(4, 2, 64, dtype=BF, device="cuda").transpose(0, 1)
    assert torch.equal(run(ea, y, out=out), want)


def test_again_and_workspace(ea):
    x = make([300, 5, 77], 500, 300, 8, 2, 128, BF, seed=7)
    want = run(ea, x)
    n = ea.prefix_decode_workspace(x["q"], x["k"], 500)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")  # NaN where nothing is written
    for _ in range(2):
        assert torch.equal(run(ea, x, workspace=ws), want)


def test_captured_and_two_streams(ea):
    x = make([300, 5, 77], 500, 300, 8, 2, 128, BF, seed=8)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(ea, x)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = run(ea, x)
    for turn, lengths in enumerate(([300, 5, 77], [0, 300, 299], [1, 1, 64])):
        new = make(lengths, 500, 300, 8, 2, 128, BF, seed=60 + turn)
        for n in x:
            x[n].copy_(new[n])
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(torch.cuda.Stream()):
            want = run(ea, new)
        torch.cuda.synchronize()
        assert torch.equal(got, want), turn


def test_a_layer(ea):
    """A prompt and a decoding step as a model makes them: norm and rotation,
    packed attention of the shared prompt and its gradients, then one more
    token of each request against the prompt's keys and its own."""
    n, B, hq, hk, d, pairs = 150, 3, 4, 2, 64, 32
    g = torch.Generator().manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=g).cuda()
    freqs = (10000.0 ** (-torch.arange(pairs) / pairs)).float().cuda()
    wq, wk = (0.5 + torch.rand(d, generator=g)).cuda(), (0.5 + torch.rand(d, generator=g)).cuda()
    q0, k0, v, do = r(n, hq, d), r(n, hk, d), r(n, hk, d), r(n, hq, d)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    q, k = ea.norm_rotary(q0, k0, pos, freqs, wq, wk)
    plan = ea.packed_plan(torch.tensor([0, n], dtype=torch.int32, device="cuda"), n)
    o, res = ea.packed_forward(q, k, v, plan)
    dq, dk, dv = ea.packed_backward(q, k, v, do, res)
    dq0, dk0, dwq, dwk = ea.norm_rotary_backward(dq, dk, q0, k0, pos, freqs, wq, wk)
    args = (pos, freqs, (pairs,), 1e-6, False)
    q64, k64 = (rotary64(t, w, *args)[0] for t, w in ((q0, wq), (k0, wk)))
    want = packed64(q64, k64, v, [0, n], 1.5, d ** -0.5, True, do)
    check("o", o, want[0], 1e-4)
    check("dv", dv, want[3], 1e-4)
    for name, t, w, up, dx, dw in (("q", q0, wq, want[1], dq0, dwq), ("k", k0, wk, want[2], dk0, dwk)):
        _, dx64, dw64 = rotary64(t, w, *args, up)
        check("d" + name, dx, dx64, 1e-4)
        check("dw" + name, dw, dw64, 1e-3)
    # one token of each request behind the prompt
    qn0, kn0, vn = r(B, hq, d), r(B, hk, d), r(B, hk, d)
    at = torch.full((B,), n, dtype=torch.int32, device="cuda")
    k_cache, v_cache = torch.zeros(B, 4, hk, d, device="cuda"), torch.zeros(B, 4, hk, d, device="cuda")
    qn, _ = ea.norm_rotary(qn0, kn0, at, freqs, wq, wk, k_out=k_cache[:, 0])
    v_cache[:, 0] = vn
    lengths = torch.ones(B, dtype=torch.int32, device="cuda")
    got = ea.prefix_decode(qn, k_cache, v_cache, lengths, k, v)
    for b in range(B):  # the same token as the prompt's last
        row = lambda a, t: torch.cat([a, t[b:b + 1].to(a)])
        x = [rotary64(row(p, t), w, torch.arange(n + 1, dtype=torch.int32), *args[1:])[0]
             for p, t, w in ((q0, qn0, wq), (k0, kn0, wk))]
        full = packed64(*x, row(v, vn), [0, n + 1], 1.5, d ** -0.5, True)[0]
        check("token %d" % b, got[b], full[-1], 1e-4)
