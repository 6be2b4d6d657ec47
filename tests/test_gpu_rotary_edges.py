"""norm_rotary_backward without tokens, through the C entry point."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_weights_gradients_of_no_tokens():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_12082_amd as ea
    r = ea.Rotary(0, 4, 2, 64, ea.EA_BF16, ea.EA_F32, 64, 0, 1, (ctypes.c_int32 * 4)(32), 1e-6)
    n = ctypes.c_size_t()
    assert ea._lib.entmax_norm_rotary_workspace(ctypes.byref(r), ctypes.byref(n)) == ea.EA_OK
    x = torch.zeros(64, device="cuda")  # something that is not null
    st = ctypes.byref(ea.Strides(0, 64))
    for which in (0, 1, 2):  # both, and each alone
        dw = [torch.full((64,), 7.0, device="cuda") for _ in range(2)]
        ptr = [None if which == 2 - i else t.data_ptr() for i, t in enumerate(dw)]
        p = x.data_ptr()
        assert ea._lib.entmax_norm_rotary_bwd(ctypes.byref(r), p, st, p, st, p, st, p, st, p, 0, p, p, p, p, p, *ptr,
                                              None, 0, torch.cuda.current_stream().cuda_stream) == ea.EA_OK
        for t, given in zip(dw, ptr):
            assert (t == (0.0 if given else 7.0)).all()
