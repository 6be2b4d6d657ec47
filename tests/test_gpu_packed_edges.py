"""Packed attention where its paths meet: the precision of dV by products,
sequences that are left out, many sequences, more tiles than workgroups,
dense query blocks among listed ones, scores that are not finite."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import HALF_STEP, check, packed64  # noqa: E402
from test_gpu_packed import ea, make, run  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("d,hq,hk", [(64, 4, 2), (128, 4, 1)])
@pytest.mark.parametrize("lists", [True, False])
def test_dv_holds_p_in_two_terms(ea, d, hq, hk, lists):
    """dV = sum p dO from p of 16 bits and more, listed or not: half a step of
    the output, 2^-15 of sum p |dO| (two bf16 terms or their like, with room),
    and 1e-4 for thresholds solved to 1e-6 (|dp| <= 2 sqrt(p) 1e-6, some hundred
    rows of |dO| <= 5, sqrt(p) <= 0.1 on average: under 1e-4)."""
    cu, tokens = [0, 700, 1500], 1500
    q, k, v, do, cud = make(cu, tokens, hq, hk, d, BF, seed=21)
    plan = ea.packed_plan(cud, tokens)
    o, res = ea.packed_forward(q, k, v, plan, alpha=1.5, tol=1e-6, max_iter=30, lists=lists)
    assert (res.lists is not None) == lists
    dv = ea.packed_backward(q, k, v, do, res)[2]
    _, _, _, want, dv_abs = packed64(q, k, v, cu, 1.5, d ** -0.5, True, do)
    check("dv d%d lists %s" % (d, lists), dv, want, 1e-4, dv_abs * 2.0 ** -15)


@pytest.mark.parametrize("hq,hk,d,dtype", [(4, 2, 64, BF), (4, 1, 128, BF), (2, 2, 128, BF), (4, 2, 64, F32)])
@pytest.mark.parametrize("causal", [True, False])
def test_sequences_that_are_left_out(ea, hq, hk, d, dtype, causal):
    """Too long, backwards, overlapping or outside: NaN in tensors that the
    calls make, the rows of no sequence 0, the others as by themselves."""
    tokens = 400
    q, k, v, do, _ = make([0, 1], tokens, hq, hk, d, dtype, seed=22)
    for cu, fine in (([5, 40, 120, 190, 390], [(5, 40), (120, 190)]),    # the second and the last are too long
                     ([0, 100, 130, 390, 400], [(100, 130), (390, 400)]),  # the first is, and the third
                     ([3, 60, 30, 90, 380], [(3, 60)]),                    # backwards, then over rows of the first
                     ([10, 200, 399], []),                                 # none is left
                     ([0, 50, 500, 80, 120], [(0, 50), (80, 120)])):       # one ends outside
        cud = torch.tensor(cu, dtype=torch.int32, device="cuda")
        plan = ea.packed_plan(cud, tokens, max_seqlen=70, causal=causal)
        got = run(ea, q, k, v, do, plan, 1.5)
        left = torch.ones(tokens, dtype=torch.bool, device="cuda")
        for a, b in fine:
            alone = torch.tensor([0, b - a], dtype=torch.int32, device="cuda")
            want = run(ea, *(t[a:b] for t in (q, k, v, do)), ea.packed_plan(alone, b - a, causal=causal), 1.5)
            left[a:b] = False
            for x, y in zip(got, want):  # (alone in other parts: sums in another order)
                check("%s %d" % (cu, a), x[a:b], y.double().cpu(), 1e-4, 2.0 ** -7 * y.double().cpu().abs())
        inside = torch.zeros_like(left)
        inside[cu[0]:cu[-1]] = True
        for x in got:
            assert torch.isnan(x[left & inside]).all(), cu
            assert not x[left & ~inside].any(), cu
        # given tensors keep their rows of no sequence, and those of the others in O
        out = torch.full_like(q, 3.0)
        grads = [torch.full_like(t, 5.0) for t in (q, k, v)]
        _, res = ea.packed_forward(q, k, v, plan, alpha=1.5, out=out)
        ea.packed_backward(q, k, v, do, res, *grads)
        assert (out[left] == 3.0).all()
        for x, y in zip([out] + grads, got):
            assert torch.equal(x[~left], y[~left])
            assert (x[left & ~inside] == (3.0 if x is out else 5.0)).all()


def test_thousands_of_sequences(ea):
    """Every row in the place that its sequence gives it, at 20000 sequences: with
    one key a sequence's rows are V itself, so every sequence is checked."""
    g = torch.Generator().manual_seed(25)
    lens = torch.randint(0, 4, (20000,), generator=g)
    lens[[7, 9999, 19999]] = torch.tensor([300, 65, 128])
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    tokens = int(cu[-1])
    q, k, v, do, _ = make([0, 1], tokens, 2, 1, 64, BF, c=2.0, seed=26)
    plan = ea.packed_plan(cu.int().cuda(), tokens, max_seqlen=300)
    got = run(ea, q, k, v, do, plan, 1.5)
    first = cu[:-1][lens > 0].cuda()  # causal: a first row sees itself alone
    assert torch.equal(got[0][first], v[first].expand(-1, 2, -1))
    for s in [7, 9999, 19999] + list(range(0, 20000, 997)):
        a, b = int(cu[s]), int(cu[s + 1])
        if a == b:
            continue
        want = packed64(q[a:b], k[a:b], v[a:b], [0, b - a], 1.5, 0.125, True, do[a:b])
        for name, x, y in zip(("o", "dq", "dk"), got, want):
            check("%d %s" % (s, name), x[a:b], y, 4e-3)
        check("%d dv" % s, got[3][a:b], want[3], 1e-3, want[4] * HALF_STEP[BF])


@pytest.mark.parametrize("alpha", [1.5, 1.7])
def test_more_tiles_than_workgroups(ea, alpha):
    """fp32 at d = 128, whose solver runs fewer workgroups at a time than there
    are tiles here (640), against the batched path: both solve to 1e-6 and are
    off by 2^-24 sqrt(d + n) |x| beside that."""
    B, n, hq, hk, d = 2, 2048, 20, 5, 128
    cu = [0, n, 2 * n]
    q, k, v, _, cud = make(cu, B * n, hq, hk, d, F32, c=2.0, seed=27)
    o, _ = ea.packed_forward(q, k, v, ea.packed_plan(cud, B * n, max_seqlen=n), alpha=alpha, need_bwd=False)
    batched = lambda t, rep: t.view(B, n, -1, d).transpose(1, 2).repeat_interleave(rep, 1).contiguous()
    want, _ = ea.forward(batched(q, 1), batched(k, 4), batched(v, 4), alpha=alpha, causal=True, need_bwd=False, tol=1e-6)
    check("a%g" % alpha, o, want.transpose(1, 2).reshape(B * n, hq, d).double().cpu(), 1e-4)


def test_dense_blocks_among_listed(ea):
    """A key head that visits more than 64 query blocks, a few of them (under an
    eighth) not listed, against the same without lists."""
    n, d, hq, hk = 5000, 128, 4, 2
    q, k, v, do, cud = make([0, n], n, hq, hk, d, BF, c=4.0, seed=23)
    for h, blocks in ((0, (3, 40, 66, 70)), (1, ()), (2, (65,)), (3, (10, 77))):
        for b in blocks:
            q[64 * b:64 * b + 64, h] *= 0.02
    plan = ea.packed_plan(cud, n)
    o, res = ea.packed_forward(q, k, v, plan, alpha=1.5)
    blocks = n // 64 + 1
    use = res.lists[-4 * hq * blocks:].view(torch.int32).view(hq, blocks)[:, :(n + 63) // 64]
    missing = ((use & 4) == 0).sum(1)
    print("blocks not listed for dK and dV, of %d: %s" % (use.shape[1], missing.tolist()), flush=True)
    assert (8 * missing <= use.shape[1]).all() and missing[0] >= 4 and missing[2] >= 1
    got = (o,) + ea.packed_backward(q, k, v, do, res)
    o, res = ea.packed_forward(q, k, v, plan, alpha=1.5, lists=False)
    want = (o,) + ea.packed_backward(q, k, v, do, res)
    for name, x, y in zip(("o", "dq", "dk", "dv"), got, want):
        # (half a step each, and gradients of scores four times as large: see test_gpu_packed)
        y = y.double().cpu()
        check(name, x, y, 1e-3 * 16, 2.0 ** -8 * y.abs())


@pytest.mark.parametrize("d,dtype", [(64, BF), (128, BF), (64, F32)])
@pytest.mark.parametrize("n", [60, 700, 1300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_scores_that_are_not_finite(ea, n, bad, d, dtype):
    """A query that is not finite, in one element (scores of +-inf, or NaN) or in
    all (NaN): its row of O is 0, the others are unchanged."""
    q, k, v, _, cud = make([0, n], n, 2, 1, d, dtype, seed=24)
    plan = ea.packed_plan(cud, n)
    want = ea.packed_forward(q, k, v, plan, alpha=1.5, need_bwd=False)[0]
    q = q.clone()
    q[n // 2, 1] = bad
    q[n // 3, 0, 5] = bad
    got = ea.packed_forward(q, k, v, plan, alpha=1.5, need_bwd=False)[0]
    assert not got[n // 2, 1].any() and not got[n // 3, 0].any()
    got[n // 2, 1], got[n // 3, 0] = want[n // 2, 1], want[n // 3, 0]
    check("n%d %s" % (n, bad), got, want.double().cpu(), 1e-4, 2.0 ** -8 * want.double().cpu().abs())
