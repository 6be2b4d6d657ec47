"""alpha > 2, where f is not convex: the thresholds of every row of a tile, whose
rows converge after different numbers of steps."""
import pytest

import synth
from gpu_util import log, to_device

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4, 70, 700, 1100])
@pytest.mark.parametrize("alpha", [2.5, 3.0])
@pytest.mark.parametrize("cached", [True, False])
def test_every_row_converges(n, alpha, cached):
    """sum p = 1 at the returned thresholds, in 64 bits.  The solver stops at
    |f| <= 1e-5; a score off by 1e-6 puts p of the key nearest to the threshold
    off by at most 1e-6^gamma (1e-3 at alpha = 3, 1e-4 at 2.5)."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_12082_amd as ea
    inp = synth.attention_inputs(1, 2, n, 64, c=1.0, dtype="bf16", seed=77)
    q, k, v = (to_device(inp[x]) for x in ("q", "k", "v"))
    _, res = ea.forward(q, k, v, alpha=alpha, causal=True, need_bwd=False, max_iter=64,
                        workspace=None if cached else False)
    x = (alpha - 1.0) * 0.125 * (q[0].double() @ k[0].double().transpose(1, 2).contiguous())
    x.masked_fill_(torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1), -float("inf"))
    z = (x - res.tau.double().view(2, n, 1)).clamp_min(0.0)
    f = (z ** (1.0 / (alpha - 1.0))).sum(-1) - 1.0
    log("alpha %g n %d: max |sum p - 1| %.3g" % (alpha, n, f.abs().max().item()))
    assert f.abs().max().item() <= 2e-3
