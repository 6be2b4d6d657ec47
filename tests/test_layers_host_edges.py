"""Sizes and objects of the calls on [tokens, heads, d] tensors (no GPU needed)."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")


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
