"""norm_rotary and its backward against the definition in 64 bits.

Tolerances beside each output's rounding: r, the rotation and the products are
some ten fp32 operations (10 x 2^-24 relative to the largest value, under 1e-5
for these inputs); a weight's gradient adds tokens x heads terms of about 1 in
fp32, each off by 1e-6, in chunks: 2e-6 sqrt(terms) + 1e-6 of the sum."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import check, rotary64  # noqa: E402

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def ea():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_12082_amd
    return paper_2502_12082_amd


def make(tokens, hq, hk, d, dtype, axes=1, pairs=None, wtype=None, seed=0, far=0):
    g = torch.Generator().manual_seed(seed)
    x = {n: (2 * torch.randn(tokens, h, d, generator=g)).to(dtype).cuda()
         for n, h in (("q", hq), ("k", hk), ("dq", hq), ("dk", hk))}
    pairs = d // 2 if pairs is None else pairs
    for n in ("q_weight", "k_weight"):
        x[n] = None if wtype is None else (0.5 + torch.rand(d, generator=g)).to(wtype).cuda()
    x["freqs"] = (10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / max(pairs, 1))).float().cuda()
    pos = torch.randint(0, 1000, (axes, tokens), generator=g, dtype=torch.int32) + far
    x["positions"] = (pos[0] if axes == 1 else pos).cuda().contiguous()
    side = pairs * 3 // 8
    x["sections"] = (pairs,) if axes == 1 else (pairs - 2 * side, side, side) if axes == 3 else (pairs, 0)
    return x


def run(ea, x, **kw):
    args = dict(q_weight=x["q_weight"], k_weight=x["k_weight"], sections=x["sections"], **kw)
    y = ea.norm_rotary(x["q"], x["k"], x["positions"], x["freqs"], **args)
    return y + ea.norm_rotary_backward(x["dq"], x["dk"], x["q"], x["k"], x["positions"], x["freqs"], **args)


def compare(got, x, eps=1e-6, interleaved=False):
    for i, n in enumerate(("q", "k")):
        y, dx, dw = rotary64(x[n], x[n + "_weight"], x["positions"], x["freqs"], x["sections"], eps, interleaved,
                             x["d" + n])
        check(n, got[i], y, 1e-5)
        # (ten operations, 2^-24 of the largest value each: with a row of zeros, r = eps^-1/2 = 32 makes
        # values of 4 x 1.5 x 32 and more, where 1e-5 is two operations' worth)
        check("d" + n, got[2 + i], dx, max(1e-5, 10 * 2.0 ** -24 * float(dx.abs().max())))
        if x[n + "_weight"] is None:
            assert got[4 + i] is None
        else:
            terms = x[n].shape[0] * x[n].shape[1]
            check("dw" + n, got[4 + i], dw, 2e-6 * terms ** 0.5 + 1e-6 * float(dw.abs().max()) + 1e-5)


@pytest.mark.parametrize("tokens", [1, 5, 259])
@pytest.mark.parametrize("hq,hk,d,dtype,wtype", [(4, 2, 64, BF, BF), (9, 3, 128, BF, F32), (3, 1, 64, F32, F32),
                                                 (17, 1, 128, F32, None), (1, 1, 128, BF, None)])
@pytest.mark.parametrize("axes,pairs,interleaved", [(1, None, False), (3, None, False), (1, None, True), (1, 8, False),
                                                    (3, 24, True), (2, 16, False), (1, 0, False)])
def test_against_definition(ea, tokens, hq, hk, d, dtype, wtype, axes, pairs, interleaved):
    x = make(tokens, hq, hk, d, dtype, axes, pairs, wtype, seed=tokens + hq)
    compare(run(ea, x, interleaved=interleaved), x, interleaved=interleaved)


def test_far_positions(ea):
    """Positions up to 2^31 - 1, and negative ones."""
    for far in (2 ** 31 - 1001, -2 ** 31):
        x = make(40, 2, 2, 64, F32, wtype=F32, far=far, seed=3)
        compare(run(ea, x), x)


def test_many_tokens(ea):
    """More tokens than waves of the backward, an eps that counts, zero rows."""
    x = make(9001, 3, 2, 64, F32, wtype=F32, seed=4)
    x["q"][17] = 0
    x["k"][:, 1] *= 1e-4
    compare(run(ea, x, eps=1e-3), x, eps=1e-3)


def test_strides_and_in_place(ea):
    tokens, hq, hk, d = 70, 4, 2, 64
    x = make(tokens, hq, hk, d, BF, wtype=BF, seed=5)
    want = run(ea, x)
    fused = torch.zeros(tokens, (hq + 2 * hk) * d, dtype=BF, device="cuda")
    q, k = fused[:, :hq * d].view(tokens, hq, d), fused[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
    q.copy_(x["q"])
    k.copy_(x["k"])
    y = dict(x, q=q, k=k, dq=x["dq"].transpose(0, 1).contiguous().transpose(0, 1))
    for a, b in zip(run(ea, y), want):
        assert torch.equal(a, b)
    args = dict(q_weight=x["q_weight"], k_weight=x["k_weight"], sections=x["sections"])
    out = ea.norm_rotary(q, k, x["positions"], x["freqs"], q_out=q, k_out=k, **args)
    assert out[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert not fused[:, (hq + hk) * d:].any()
    apart = torch.zeros(hq, tokens, d, dtype=BF, device="cuda").transpose(0, 1)
    ea.norm_rotary(x["q"], x["k"], x["positions"], x["freqs"], q_out=apart, **args)
    assert torch.equal(apart, want[0])


def test_no_tokens(ea):
    x = make(0, 2, 1, 64, BF, wtype=F32)
    got = run(ea, x)
    assert got[0].shape == (0, 2, 64) and got[2].shape == (0, 2, 64)
    assert not got[4].any() and not got[5].any()


def test_differences(ea):
    x = make(30, 3, 2, 64, F32, wtype=F32, seed=6)
    args = (x["positions"], x["freqs"])
    grads = run(ea, x)[2:]

    def loss(q, k, wq, wk):
        a, b = ea.norm_rotary(q, k, *args, q_weight=wq, k_weight=wk)
        return float((a.double() * x["dq"].double()).sum() + (b.double() * x["dk"].double()).sum())

    base = [x["q"], x["k"], x["q_weight"], x["k_weight"]]
    g = torch.Generator().manual_seed(1)
    for i, t in enumerate(base):
        step = torch.randn(t.shape, generator=g).cuda() / t.numel() ** 0.5
        h = 1e-2
        ends = [loss(*[y + (s * h * step if j == i else 0) for j, y in enumerate(base)]) for s in (1, -1)]
        diff, want = (ends[0] - ends[1]) / (2 * h), float((grads[i].double() * step.double()).sum())
        print(i, diff, want, flush=True)
        # 9600 outputs off by about 2^-23 each, times their gradients of 2 rms: 2e-5 on either end, so
        # 1.4e-3 rms after the division by 2 h; four times that
        assert abs(diff - want) <= 6e-3 * max(1.0, abs(want))


def test_captured(ea):
    x = make(300, 4, 2, 128, BF, wtype=BF, seed=7)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(ea, x)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = run(ea, x)
    for turn in range(3):
        new = make(300, 4, 2, 128, BF, wtype=BF, seed=50 + turn)
        for n in ("q", "k", "dq", "dk", "positions", "q_weight", "k_weight"):
            x[n].copy_(new[n])
        graph.replay()
        torch.cuda.synchronize()
        want = run(ea, new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn
