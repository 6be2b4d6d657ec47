"""Packed alpha-entmax attention with grouped heads, forward and backward,
against the definition in 64 bits.

Tolerances.  Beside the rounding of each output (half a step of its type):
fp32 accumulation of up to a few hundred products of N(0, 1) values is off by
under 2^-24 sqrt(d + n) |x| < 1e-5, and the threshold by the solver's tolerance
(1e-5, fp32 1e-6) times |v| <= 5; p, u and dS enter their products as two bf16
terms (2^-16 relative).  Gradients carry the factor |dP| <~ 50 on the error of
u, which is that of z (1e-6) for gamma = 2: 1e-3 for bf16 covers it, 1e-4 for
fp32.  For a general alpha above 1.5 the slope of u, z^(gamma-2), has no bound:
the nearest of 10^4 scores to its threshold, z ~ 10^-5, has u off by 0.33
z^-0.67 10^-6 ~ 10^-3, times |dP|: 2e-2 for bf16 (fp32 inputs are scored in 64
bits there).  dV takes p rounded to bf16: half a step of sum p |dO|."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import HALF_STEP, check, packed64  # noqa: E402

pytestmark = pytest.mark.gpu
ATOL = {torch.bfloat16: 1e-3, torch.float32: 1e-4}
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def ea():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_12082_amd
    return paper_2502_12082_amd


def make(cu, tokens, hq, hk, d, dtype, c=1.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    t = [r(tokens, hq, d) * c, r(tokens, hk, d), r(tokens, hk, d), r(tokens, hq, d)]
    return [x.to(dtype).cuda() for x in t] + [torch.tensor(cu, dtype=torch.int32, device="cuda")]


def run(ea, q, k, v, do, plan, alpha, **kw):
    o, res = ea.packed_forward(q, k, v, plan, alpha=alpha, **kw)
    return (o,) + ea.packed_backward(q, k, v, do, res)


def compare(got, q, k, v, do, cu, alpha, causal, label, c=1.0):
    d = q.shape[-1]
    o, dq, dk, dv, dv_abs = packed64(q, k, v, cu, alpha, d ** -0.5, causal, do)
    # queries c times as large: so are the scores' roundings, which u takes over, and the q that dK multiplies it with
    atol = (2e-2 if alpha == 1.75 else ATOL[q.dtype]) * max(1.0, c * c)
    operand = dv_abs * (HALF_STEP[BF] if q.dtype == BF else 0.0)
    for name, x, want, extra in (("o", got[0], o, None), ("dq", got[1], dq, None), ("dk", got[2], dk, None),
                                 ("dv", got[3], dv, operand)):
        check(label + " " + name, x, want, atol, extra)


LENGTHS = {
    "one": ([0, 1], 1),
    "block": ([0, 64], 64),
    "edges": ([0, 65, 66, 129, 257, 259], 259),
    "empty": ([0, 0, 70, 70, 70, 90, 90], 90),
    "rest": ([3, 40, 180], 191),  # rows of no sequence on both sides
    "longer": ([0, 300, 317, 700], 700),
}


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hk,d,dtype,alpha", [
    (4, 2, 64, BF, 1.5), (6, 2, 128, BF, 1.5), (4, 1, 64, F32, 1.5), (2, 2, 128, F32, 1.25),
    (3, 3, 128, BF, 1.25), (4, 4, 64, BF, 1.75), (3, 1, 64, F32, 1.7)])
def test_against_definition(ea, lengths, causal, hq, hk, d, dtype, alpha):
    cu, tokens = LENGTHS[lengths]
    q, k, v, do, cud = make(cu, tokens, hq, hk, d, dtype, seed=len(lengths) + hq)
    plan = ea.packed_plan(cud, tokens, causal=causal)
    got = run(ea, q, k, v, do, plan, alpha)
    compare(got, q, k, v, do, cu, alpha, causal, "%s %s %d/%d d%d a%g" % (lengths, dtype, hq, hk, d, alpha))
    outside = torch.ones(tokens, dtype=torch.bool)
    for a, b in zip(cu[:-1], cu[1:]):
        outside[a:b] = False
    for x in got:
        assert not x[outside.cuda()].any()


@pytest.mark.parametrize("alpha", [2.0, 1.6, 2.5])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_forward_other_exponents(ea, alpha, dtype):
    """alpha = 2 (whose gradient jumps at the support's edge) and general alpha, forward."""
    cu, tokens = [0, 5, 150, 400], 400
    q, k, v, _, cud = make(cu, tokens, 4, 2, 64, dtype, seed=5)
    o, res = ea.packed_forward(q, k, v, ea.packed_plan(cud, tokens), alpha=alpha, need_bwd=False, max_iter=40)
    check("o", o, packed64(q, k, v, cu, alpha, 64 ** -0.5, True)[0], ATOL[dtype])
    with pytest.raises(ValueError):
        ea.packed_backward(q, k, v, q, res)


@pytest.mark.parametrize("c", [0.05, 30.0])
def test_dense_and_one_hot_rows(ea, c):
    """Rows with every key in the support, and rows of one key."""
    cu, tokens = [0, 500, 530], 530
    q, k, v, do, cud = make(cu, tokens, 4, 2, 128, BF, c=c, seed=9)
    got = run(ea, q, k, v, do, ea.packed_plan(cud, tokens), 1.5)
    # a one-hot row's z carries the rounding of scores c times as large
    o, dq, dk, dv, dv_abs = packed64(q, k, v, cu, 1.5, 128 ** -0.5, True, do)
    atol = 1e-3 * max(1.0, c)
    for name, x, want, extra in (("o", got[0], o, None), ("dq", got[1], dq, None), ("dk", got[2], dk, None),
                                 ("dv", got[3], dv, dv_abs * HALF_STEP[BF])):
        check("c%g %s" % (c, name), x, want, atol, extra)


@pytest.mark.parametrize("d,hq,hk", [(64, 8, 2), (128, 16, 8)])
def test_equals_the_batched_path(ea, d, hq, hk):
    """A batch of equal lengths, packed, against forward and backward on
    [B, H, n, d] (the 128 case adds up its query heads in one workgroup)."""
    B, n = 4, 2048
    tokens = B * n
    cu = [i * n for i in range(B + 1)]
    q, k, v, do, cud = make(cu, tokens, hq, hk, d, BF, c=2.0, seed=3)
    got = run(ea, q, k, v, do, ea.packed_plan(cud, tokens, max_seqlen=n), 1.5)
    batched = lambda t, rep: t.view(B, n, -1, d).transpose(1, 2).repeat_interleave(rep, 1).contiguous()
    g = hq // hk
    qb, kb, vb, dob = batched(q, 1), batched(k, g), batched(v, g), batched(do, 1)
    o, res = ea.forward(qb, kb, vb, alpha=1.5, causal=True)
    dq, dk, dv = ea.backward(qb, kb, vb, dob, res)
    back = lambda t, heads: t.float().view(B, heads, -1, n, d).sum(2).transpose(1, 2).reshape(tokens, heads, d)
    # sum p |dO|, which half a step of a rounded p multiplies: dV is linear in dO
    dv_abs = back(ea.backward(qb, kb, vb, dob.abs(), res)[2], hk).double().cpu()
    for name, x, want in (("o", got[0], back(o, hq)), ("dq", got[1], back(dq, hq)), ("dk", got[2], back(dk, hk)),
                          ("dv", got[3], back(dv, hk))):
        # two roundings of o, one of the gradients, two of p in dV (either path may round it); thresholds
        # solved to 1e-5 on either side
        extra = 2.0 ** -7 * dv_abs if name == "dv" else 2.0 ** -8 * want.double().cpu().abs()
        check(name, x, want.double().cpu(), 2e-3, extra)


def test_many_sequences(ea):
    """More sequences than a wave has lanes, most of a few rows, one long."""
    g = torch.Generator().manual_seed(11)
    lens = torch.randint(0, 12, (700,), generator=g).tolist()
    lens[300] = 4200
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    tokens = cu[-1]
    q, k, v, do, cud = make(cu, tokens, 2, 1, 64, BF, c=2.0, seed=12)
    got = run(ea, q, k, v, do, ea.packed_plan(cud, tokens, max_seqlen=4200), 1.5)
    sub = [s for s in range(700) if s != 300 and lens[s]][::9]
    for s in sub:
        a, b = cu[s], cu[s + 1]
        o, dq, dk, dv, dv_abs = packed64(q[a:b], k[a:b], v[a:b], [0, b - a], 1.5, 0.125, True, do[a:b])
        check("seq %d o" % s, got[0][a:b], o, 1e-3)
        check("seq %d dq" % s, got[1][a:b], dq, 1e-3)
        check("seq %d dk" % s, got[2][a:b], dk, 1e-3)
        check("seq %d dv" % s, got[3][a:b], dv, 1e-3, dv_abs * HALF_STEP[BF])
    a, b = cu[300], cu[301]
    alone = torch.tensor([0, 4200], dtype=torch.int32, device="cuda")
    want = run(ea, *(t[a:b] for t in (q, k, v, do)), ea.packed_plan(alone, 4200), 1.5)
    for x, y in zip(got, want):  # the same sequence by itself (in other parts: sums in another order)
        check("long", x[a:b], y.double().cpu(), 1e-3, 2.0 ** -8 * y.double().cpu().abs())


def test_strides(ea):
    """Slices of a fused projection, head-major tensors, padded rows."""
    cu, tokens, hq, hk, d = [0, 100, 230], 230, 4, 2, 64
    g = torch.Generator().manual_seed(2)
    fused = torch.randn(tokens, (hq + 2 * hk) * d + 8, generator=g).to(BF).cuda()
    q = fused[:, :hq * d].view(tokens, hq, d)
    k = fused[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
    v = torch.randn(hk, tokens, d, generator=g).to(BF).cuda().transpose(0, 1)
    do = torch.randn(hq, tokens, 2 * d, generator=g).to(BF).cuda()[..., :d].transpose(0, 1)
    plan = ea.packed_plan(torch.tensor(cu, dtype=torch.int32, device="cuda"), tokens)
    want = run(ea, *(t.contiguous() for t in (q, k, v, do)), plan, 1.5)
    out = torch.full((hq, tokens, d), 7.0, dtype=BF, device="cuda").transpose(0, 1)
    o, res = ea.packed_forward(q, k, v, plan, alpha=1.5, out=out)
    assert o is out
    for x, y in zip((o,) + ea.packed_backward(q, k, v, do, res), want):
        assert torch.equal(x, y)


def test_rows_of_no_sequence_stay(ea):
    cu, tokens = [2, 60, 133], 150
    q, k, v, do, cud = make(cu, tokens, 4, 2, 128, BF, seed=4)
    for t in (q, k, v, do):  # what those rows hold reaches nothing
        t[:2] = float("nan")
        t[133:] = float("inf")
    plan = ea.packed_plan(cud, tokens)
    want = run(ea, q, k, v, do, plan, 1.5)
    out = torch.full_like(q, 3.0)
    grads = [torch.full_like(t, 5.0) for t in (q, k, v)]
    _, res = ea.packed_forward(q, k, v, plan, alpha=1.5, out=out)
    ea.packed_backward(q, k, v, do, res, *grads)
    for x, y, fill in zip([out] + grads, want, (3.0, 5.0, 5.0, 5.0)):
        assert torch.equal(x[2:133], y[2:133]) and not torch.isnan(y).any()
        assert (x[:2] == fill).all() and (x[133:] == fill).all()
        assert (y[:2] == 0).all() and (y[133:] == 0).all()


def test_sequences_that_are_none(ea):
    """Ranges that overlap, run backwards, leave the tensors or are too long are
    left out, and the others are computed."""
    tokens = 300
    cu = [0, 40, 20, 90, 400, 290, 300]
    q, k, v, do, cud = make(cu, tokens, 2, 2, 64, BF, seed=6)
    got = run(ea, q, k, v, do, ea.packed_plan(cud, tokens, max_seqlen=60), 1.5)
    for a, b in ((0, 40), (290, 300)):
        want = packed64(q[a:b], k[a:b], v[a:b], [0, b - a], 1.5, 0.125, True, do[a:b])
        check("o", got[0][a:b], want[0], 1e-3)
        check("dq", got[1][a:b], want[1], 1e-3)


def test_without_workspace_and_again(ea):
    """The solver without its cache, and bit-equal results of a second call."""
    cu, tokens = [0, 700, 1500], 1500
    q, k, v, do, cud = make(cu, tokens, 4, 2, 64, BF, c=2.0, seed=7)
    plan = ea.packed_plan(cud, tokens)
    first, again = run(ea, q, k, v, do, plan, 1.5), run(ea, q, k, v, do, plan, 1.5)
    for x, y in zip(first, again):
        assert torch.equal(x, y)
    # (thresholds solved to 1e-5 on either side; p, rounded in dV or, from element lists, not)
    dv_abs = run(ea, q, k, v, do.abs(), plan, 1.5)[3].double().cpu()
    small = torch.empty(3 * 1179648 + 7, dtype=torch.uint8, device="cuda")  # three cache slots
    for name, ws in (("no workspace", False), ("small workspace", small)):
        for i, (x, y) in enumerate(zip(run(ea, q, k, v, do, plan, 1.5, workspace=ws), first)):
            y = y.double().cpu()
            check(name, x, y, 1e-3, 2.0 ** -7 * dv_abs if i == 3 else 2.0 ** -8 * y.abs())


@pytest.mark.parametrize("d,dtype,alpha,c", [(64, BF, 1.5, 3.0), (128, BF, 1.25, 6.0), (128, BF, 1.5, 1.0),
                                             (64, F32, 1.5, 2.0), (128, F32, 1.7, 3.0)])
@pytest.mark.parametrize("causal", [True, False])
def test_element_lists(ea, d, dtype, alpha, c, causal):
    """Sparse rows, whose blocks are listed, against the same call without lists
    and the definition; some sequences short, some dense enough to be not listed."""
    cu, tokens = [0, 640, 650, 1400, 1500], 1500
    q, k, v, do, cud = make(cu, tokens, 4, 2, d, dtype, c=c, seed=14)
    q[650:1000] *= 0.1
    plan = ea.packed_plan(cud, tokens, causal=causal)
    o, res = ea.packed_forward(q, k, v, plan, alpha=alpha)
    blocks = 4 * (tokens // 64 + 4)
    use = res.lists[-4 * blocks:].view(torch.int32)
    assert int((use[:96] != 0).sum()) > 5, "no block is listed"
    got = (o,) + ea.packed_backward(q, k, v, do, res)
    compare(got, q, k, v, do, cu, alpha, causal, "lists d%d a%g c%g" % (d, alpha, c), c)
    small = torch.empty(res.sizes.ws_bwd, dtype=torch.uint8, device="cuda")  # no room to sort the lists
    compare((o,) + ea.packed_backward(q, k, v, do, res, workspace=small), q, k, v, do, cu, alpha, causal, "small", c)
    o, res = ea.packed_forward(q, k, v, plan, alpha=alpha, lists=False)
    assert res.lists is None
    compare((o,) + ea.packed_backward(q, k, v, do, res), q, k, v, do, cu, alpha, causal, "none", c)


@pytest.mark.parametrize("d,dtype,alpha,c", [(64, BF, 1.5, 3.0), (128, BF, 1.25, 6.0), (64, F32, 2.0, 2.0),
                                             (128, F32, 1.5, 3.0)])
@pytest.mark.parametrize("cu", [[0, 700, 710, 1000], [0, 256, 330, 587], [0, 255, 256, 300]])
def test_short_sequences(ea, cu, d, dtype, alpha, c):
    """Sequences of up to 1024, 512 and 256 keys in strided rows, listed where they are long enough."""
    n = max(b - a for a, b in zip(cu, cu[1:]))
    q, k, v, do, cud = make(cu, cu[-1], 4, 2, d, dtype, c=c, seed=17)
    wide = torch.cat([q, k, v], 1)
    q, k, v = wide[:, :4], wide[:, 4:6], wide[:, 6:]
    for causal in (True, False):
        plan = ea.packed_plan(cud, cu[-1], max_seqlen=n, causal=causal)
        got = run(ea, q, k, v, do, plan, alpha)
        compare(got, q, k, v, do, cu, alpha, causal, "short %d d%d a%g" % (n, d, alpha), c)
        assert torch.equal(got[0], ea.packed_forward(q, k, v, plan, alpha=alpha, workspace=False)[0])


def test_differences(ea):
    """Gradients against central differences of the fp32 forward.  Its 25600
    outputs are off by some 3e-7 each: 5e-5 on either end of the difference, so
    7e-4 rms after the division by 2 h; the tolerance is seven times that (the
    differences' own h^2 term, for a step of length 0.05 over all elements, is
    far below)."""
    cu, tokens = [0, 33, 100], 100
    q, k, v, do, cud = make(cu, tokens, 4, 2, 64, F32, seed=8)
    plan = ea.packed_plan(cud, tokens)
    loss = lambda a, b, c_: float((ea.packed_forward(a, b, c_, plan, alpha=1.5, tol=0.0)[0].double() * do.double()).sum())
    grads = run(ea, q, k, v, do, plan, 1.5, tol=0.0)[1:]
    g = torch.Generator().manual_seed(1)
    for i, t in enumerate((q, k, v)):
        step = torch.randn(t.shape, generator=g).cuda() / t.numel() ** 0.5
        h = 5e-2
        args = [[x + (s * h * step if j == i else 0) for j, x in enumerate((q, k, v))] for s in (1, -1)]
        diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
        want = float((grads[i].double() * step.double()).sum())
        print(i, diff, want, flush=True)
        assert abs(diff - want) <= 5e-3 * max(1.0, abs(want))


def test_captured(ea):
    """Plan, forward and backward in one graph: replayed with other inputs and
    other lengths, with eager work between the replays."""
    tokens, hq, hk, d = 600, 4, 2, 64
    q, k, v, do, cud = make([0, 100, 350, 600], tokens, hq, hk, d, BF, seed=20)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        run(ea, q, k, v, do, ea.packed_plan(cud, tokens), 1.5)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = run(ea, q, k, v, do, ea.packed_plan(cud, tokens), 1.5)
    for turn, cu in enumerate(([0, 100, 350, 600], [0, 600, 600, 600], [0, 1, 2, 570])):
        new = make(cu, tokens, hq, hk, d, BF, seed=30 + turn)
        for x, y in zip((q, k, v, do, cud), new):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        want = run(ea, *new[:4], ea.packed_plan(new[4], tokens), 1.5)
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), turn


def test_two_streams(ea):
    cu, tokens = [0, 900, 1000], 1000
    cases = [make(cu, tokens, 4, 2, 64, BF, seed=40 + i) for i in range(2)]
    want = [run(ea, *c[:4], ea.packed_plan(c[4], tokens), 1.5) for c in cases]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in cases], []
    for c, s in zip(cases, streams):
        with torch.cuda.stream(s):
            got.append(run(ea, *c[:4], ea.packed_plan(c[4], tokens), 1.5))
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(x, y))


def test_longest_sequences(ea):
    """More keys than 16 bits number, against the batched path."""
    n, d = 70001, 64
    q, k, v, _, cud = make([0, n], n, 2, 1, d, BF, c=4.0, seed=15)
    o, res = ea.packed_forward(q, k, v, ea.packed_plan(cud, n), alpha=1.5, need_bwd=False)
    assert res.lists is None
    batched = lambda t: t.transpose(0, 1)[None].contiguous()
    kk, vv = (t.repeat_interleave(2, 1) for t in (k, v))
    want, _ = ea.forward(batched(q), batched(kk), batched(vv), alpha=1.5, causal=True, need_bwd=False)
    want = want[0].transpose(0, 1).double().cpu()
    check("long", o, want, 1e-3, 2.0 ** -8 * want.abs())


def test_far_rows(ea):
    """Rows so far apart that their offsets pass 32 bits, in elements and bytes."""
    tokens, hq, hk, d, width = 20000, 2, 1, 64, 120000
    cu = [0, 19000, tokens]
    q, k, v, do, cud = make(cu, tokens, hq, hk, d, BF, c=4.0, seed=16)
    plan = ea.packed_plan(cud, tokens)
    want = run(ea, q, k, v, do, plan, 1.5)
    wide = torch.empty(tokens, width, dtype=BF, device="cuda")
    parts, at = [], 0
    for t in (q, k, v, do):
        part = wide[:, at:at + t.shape[1] * d].view(t.shape)
        part.copy_(t)
        parts.append(part)
        at += 30000
    got = run(ea, *parts, plan, 1.5)
    assert all(torch.equal(x, y) for x, y in zip(got, want))
