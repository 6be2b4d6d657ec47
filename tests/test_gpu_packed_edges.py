"""Packed attention where its paths meet: the precision of dV by products."""
import pytest

torch = pytest.importorskip("torch")
from layer_util import check, packed64  # noqa: E402
from test_gpu_packed import ea, make  # noqa: E402,F401

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


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
