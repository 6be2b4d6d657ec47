"""Sizes and objects of the calls on [tokens, heads, d] tensors (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")


SLOT = 1179648  # bytes of one cache slot of the solver


def test_solvers_that_run_at_a_time():
    """The packed solver's workgroups are those that run at a time: three on each
    of 256 compute units; fp32 at d = 128 two (68 KB of key tiles each), with a
    general alpha one (428 registers).  They take half a cache slot each."""
    z = ea.PackedSizes()
    for d, dtype, alpha, groups in ((64, ea.EA_BF16, 1.5, 768), (128, ea.EA_BF16, 1.7, 768), (64, ea.EA_F32, 1.7, 768),
                                    (128, ea.EA_F32, 1.5, 512), (128, ea.EA_F32, 1.25, 512), (128, ea.EA_F32, 2.0, 512),
                                    (128, ea.EA_F32, 1.7, 256)):
        params = ea.make_params(alpha, None, True, True, None, None, head_dim=64)
        shape = ea.PackedShape(65536, 1, 65536, 8, 8, d, dtype)
        assert ea._lib.entmax_packed_sizes(shape, ctypes.byref(params), ctypes.byref(z)) == ea.EA_OK
        assert z.ws_fwd == groups // 2 * SLOT, (d, dtype, alpha)


def test_sequences_of_a_plan():
    """plan_kernel's work grows with the square of the sequences: more than 2^16
    are refused before any launch."""
    n = ctypes.c_size_t()
    assert ea._lib.entmax_packed_plan_bytes(1000, 1 << 16, ctypes.byref(n)) == ea.EA_OK
    assert ea._lib.entmax_packed_plan_bytes(1000, (1 << 16) + 1, ctypes.byref(n)) == ea.EA_ERR_UNSUPPORTED
    params, z = ea.make_params(1.5, None, True, True, None, None, head_dim=64), ea.PackedSizes()
    size = lambda seqs: ea._lib.entmax_packed_sizes(ea.PackedShape(1000, seqs, 100, 1, 1, 64, ea.EA_BF16),
                                                    ctypes.byref(params), ctypes.byref(z))
    assert size(1 << 16) == ea.EA_OK and size((1 << 16) + 1) == ea.EA_ERR_UNSUPPORTED


def test_decoding_grid_of_one_launch():
    """Workgroups over keys that one launch cannot hold (2^26 of 64 threads) are
    refused by the sizes: 8 x 1024 for every request's own cache, and those of
    the prefix with them."""
    n = ctypes.c_size_t()
    size = lambda *s: ea._lib.entmax_prefix_decode_workspace(ea.DecodeShape(*s), ctypes.byref(n))
    assert size(8191, 8, 8, 64, ea.EA_BF16, 0, 131072) == ea.EA_OK
    assert size(8192, 8, 8, 64, ea.EA_BF16, 0, 131072) == ea.EA_ERR_UNSUPPORTED
    # 8199 x 8 x 1023 = 2^26 - 8248; 257 tiles of 32 rows, 8 key heads, one run: 2056 more; in 64 rows 1032
    assert size(8199, 8, 8, 64, ea.EA_F32, 128, 130944) == ea.EA_OK
    # 8200 x 8 x 1023 = 2^26 - 64
    assert size(8200, 8, 8, 64, ea.EA_F32, 0, 130944) == ea.EA_OK
    assert size(8200, 8, 8, 64, ea.EA_F32, 128, 130944) == ea.EA_ERR_UNSUPPORTED


def test_residuals_own_their_structures():
    """What one call's residuals hold is no other call's: the structures that the
    binding keeps for a set of sizes are not handed out."""
    plan = ea.PackedPlan(torch.zeros(4096, dtype=torch.uint8), 10, 2, 10, True)
    t = [torch.zeros(10, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)]
    key = (1.5, None, None, None, True, True, 64, 10, 2, 10, 4, 2, 64, ea.EA_BF16)

    def make():
        params, sizes = ea._packed_params(*key)
        return ea.PackedResiduals(ea._packed_shape(*t, plan), params, plan, sizes, "cpu")

    first = make()
    scale, nbytes = first.params.scale, first.sizes.ws_bwd
    first.params.scale, first.sizes.ws_bwd, first.shape.tokens = 7.0, 1, 3
    second = make()
    assert second.params.scale == scale and second.sizes.ws_bwd == nbytes and second.shape.tokens == 10
    assert ea._packed_shape(*t, plan).tokens == 10
