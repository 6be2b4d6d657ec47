"""Refusals of the calls on [tokens, heads, d] tensors, before anything is
launched (no GPU needed): by the binding, and by the C entry points."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")
BF = torch.bfloat16


def rotary_args(**kw):
    a = dict(q=torch.zeros(5, 4, 64, dtype=BF), k=torch.zeros(5, 2, 64, dtype=BF),
             positions=torch.zeros(5, dtype=torch.int32), freqs=torch.zeros(32))
    a.update(kw)
    return a


@pytest.mark.parametrize("change,word", [
    (dict(q=torch.zeros(5, 4, 64, dtype=torch.float16)), "bfloat16"),
    (dict(q=torch.zeros(5, 256, dtype=BF)), "tokens, heads"),
    (dict(k=torch.zeros(4, 2, 64, dtype=BF)), "shape"),
    (dict(k=torch.zeros(5, 2, 64)), "dtype"),
    (dict(q=torch.zeros(5, 64, 4, dtype=BF).transpose(1, 2)), "contiguous"),
    (dict(q=torch.zeros(5, 4, 68, dtype=BF)[..., :64]), "16 bytes"),
    (dict(q=torch.zeros(5 * 256 + 1, dtype=BF)[1:].view(5, 4, 64)), "16 bytes"),
    (dict(positions=torch.zeros(5, dtype=torch.int64)), "int32"),
    (dict(positions=torch.zeros(6, dtype=torch.int32)), "positions"),
    (dict(positions=torch.zeros(3, 5, dtype=torch.int32)), "positions"),
    (dict(freqs=torch.zeros(33)), "multiple of 8"),
    (dict(freqs=torch.zeros(40)), "multiple of 8"),
    (dict(freqs=torch.zeros(32, dtype=torch.float64)), "dtype"),
    (dict(sections=(16, 15)), "sections"),
    (dict(sections=(8, 8, 8, 4, 4)), "sections"),
    (dict(sections=(40, -8)), "sections"),
    (dict(q_weight=torch.zeros(63)), "shape"),
    (dict(q_weight=torch.zeros(64, dtype=torch.float64)), "weights"),
    (dict(q_weight=torch.zeros(64), k_weight=torch.zeros(64, dtype=BF)), "dtype"),
    (dict(q_out=torch.zeros(5, 4, 32, dtype=BF)), "shape"),
    (dict(q_out=torch.zeros(5, 1, 64, dtype=BF).expand(5, 4, 64)), "memory|16 bytes"),
    (dict(), "GPU"),
])
def test_norm_rotary_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        ea.norm_rotary(**rotary_args(**change))


def test_norm_rotary_refuses_overlap():
    a = rotary_args()
    base = torch.zeros(6, 4, 64, dtype=BF)
    with pytest.raises(ValueError, match="overlap"):  # one row further on
        ea.norm_rotary(**dict(a, q=base[:5], q_out=base[1:]))
    with pytest.raises(ValueError, match="overlap"):  # queries written over keys
        ea.norm_rotary(**dict(a, k=base[:5, :2], q_out=base[:5]))
    with pytest.raises(ValueError, match="GPU"):  # parts of one projection's rows: apart
        ea.norm_rotary(**dict(a, q=base[:5, :2], k=base[:5, 2:], q_out=base[:5, :2], k_out=base[:5, 2:]))


@pytest.mark.parametrize("field,value,code", [
    ("tokens", -1, ea.EA_ERR_INVALID_ARG), ("heads", 0, ea.EA_ERR_INVALID_ARG), ("head_dim", 96, ea.EA_ERR_UNSUPPORTED),
    ("dtype", 3, ea.EA_ERR_UNSUPPORTED), ("weight_dtype", 0, ea.EA_ERR_UNSUPPORTED), ("rot_dim", 24, ea.EA_ERR_INVALID_ARG),
    ("rot_dim", 144, ea.EA_ERR_INVALID_ARG), ("axes", 0, ea.EA_ERR_INVALID_ARG), ("axes", 5, ea.EA_ERR_INVALID_ARG),
    ("eps", -1.0, ea.EA_ERR_INVALID_ARG), ("eps", float("nan"), ea.EA_ERR_INVALID_ARG),
    ("interleaved", 2, ea.EA_ERR_INVALID_ARG)])
def test_norm_rotary_abi(field, value, code):
    r = ea.Rotary(5, 4, 2, 128, ea.EA_F32, ea.EA_F32, 64, 0, 1, (ctypes.c_int32 * 4)(32), 1e-6)
    n = ctypes.c_size_t()
    assert ea._lib.entmax_norm_rotary_workspace(ctypes.byref(r), ctypes.byref(n)) == ea.EA_OK and n.value > 0
    setattr(r, field, value)
    assert ea._lib.entmax_norm_rotary_workspace(ctypes.byref(r), ctypes.byref(n)) == code


def plan(tokens=10, causal=True, max_seqlen=10):
    return ea.PackedPlan(torch.zeros(4096, dtype=torch.uint8), tokens, 2, max_seqlen, causal)


def packed_args(**kw):
    a = dict(q=torch.zeros(10, 4, 64, dtype=BF), k=torch.zeros(10, 2, 64, dtype=BF), v=torch.zeros(10, 2, 64, dtype=BF),
             plan=plan())
    a.update(kw)
    return a


@pytest.mark.parametrize("change,word", [
    (dict(plan=None), "plan"),
    (dict(plan=plan(11)), "rows"),
    (dict(k=torch.zeros(10, 3, 64, dtype=BF)), "multiple"),
    (dict(v=torch.zeros(10, 4, 64, dtype=BF)), "shape"),
    (dict(v=torch.zeros(10, 2, 64)), "dtype"),
    (dict(k=torch.zeros(10, 2, 66, dtype=BF)[..., :64]), "16 bytes"),
    (dict(out=torch.zeros(10, 4, 64)), "dtype"),
    (dict(out=torch.zeros(1, 4, 64, dtype=BF).expand(10, 4, 64)), "memory"),
    (dict(workspace=torch.zeros(4).t().expand(3, 4)), "contiguous"),
    (dict(), "GPU"),
])
def test_packed_forward_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        ea.packed_forward(**packed_args(**change))


def test_packed_forward_refuses_overlap():
    a = packed_args()
    with pytest.raises(ValueError, match="overlap"):
        ea.packed_forward(**dict(a, out=a["q"]))


@pytest.mark.parametrize("alpha", [1.0, 0.5, float("nan"), float("inf")])
def test_packed_alpha(alpha):
    with pytest.raises(ea.EntmaxAttnError) as e:
        ea.packed_forward(**packed_args(alpha=alpha))
    assert e.value.status == ea.EA_ERR_INVALID_ARG


@pytest.mark.parametrize("d", [32, 96, 256])
def test_packed_head_dim(d):
    a = packed_args(q=torch.zeros(10, 4, d), k=torch.zeros(10, 2, d), v=torch.zeros(10, 2, d))
    with pytest.raises(ea.EntmaxAttnError) as e:
        ea.packed_forward(**a)
    assert e.value.status == ea.EA_ERR_UNSUPPORTED


def residuals(a, need_bwd=True):
    p = a["plan"]
    shape = ea._packed_shape(a["q"], a["k"], a["v"], p)
    params = ea.make_params(1.5, None, True, need_bwd, head_dim=64)
    sizes = ea.PackedSizes()
    ea._check(ea._lib.entmax_packed_sizes(ctypes.byref(shape), ctypes.byref(params), ctypes.byref(sizes)), "sizes")
    return ea.PackedResiduals(shape, params, p, sizes, "cpu")


@pytest.mark.parametrize("change,word", [
    (dict(res=None), "residuals"),
    (dict(dout=torch.zeros(10, 4, 64)), "dtype"),
    (dict(dout=torch.zeros(10, 2, 64, dtype=BF)), "shape"),
    (dict(q=torch.zeros(10, 2, 64, dtype=BF)), "another shape"),
    (dict(dq=torch.zeros(10, 4, 64, dtype=BF)), "together"),
    (dict(dq=torch.zeros(10, 4, 64), dk=torch.zeros(10, 2, 64, dtype=BF), dv=torch.zeros(10, 2, 64, dtype=BF)), "dtype"),
    (dict(workspace=torch.zeros(8, dtype=torch.uint8)), "workspace"),
    (dict(), "GPU"),
])
def test_packed_backward_refuses(change, word):
    a = packed_args()
    args = dict(q=a["q"], k=a["k"], v=a["v"], dout=torch.zeros(10, 4, 64, dtype=BF), res=residuals(a))
    args.update(change)
    with pytest.raises(ValueError, match=word):
        ea.packed_backward(**args)


def test_packed_backward_refuses_inference_and_overlap():
    a = packed_args()
    do = torch.zeros(10, 4, 64, dtype=BF)
    with pytest.raises(ValueError, match="need_bwd"):
        ea.packed_backward(a["q"], a["k"], a["v"], do, residuals(a, False))
    dk = torch.zeros(10, 2, 64, dtype=BF)
    with pytest.raises(ValueError, match="overlap"):
        ea.packed_backward(a["q"], a["k"], a["v"], do, residuals(a), torch.zeros_like(do), dk, dk)
    with pytest.raises(ValueError, match="overlaps dout"):
        ea.packed_backward(a["q"], a["k"], a["v"], do, residuals(a), do, dk, torch.zeros_like(dk))


@pytest.mark.parametrize("cu,kw,word", [
    (torch.zeros(1, dtype=torch.int32), {}, "at least one"),
    (torch.zeros(3, dtype=torch.int64), {}, "dtype"),
    (torch.zeros(6, dtype=torch.int32)[::2], {}, "contiguous"),
    (torch.zeros(3, dtype=torch.int32), dict(tokens=0), "tokens"),
    (torch.zeros(3, dtype=torch.int32), dict(max_seqlen=0), "max_seqlen"),
    (torch.zeros(3, dtype=torch.int32), {}, "GPU"),
])
def test_packed_plan_refuses(cu, kw, word):
    with pytest.raises(ValueError, match=word):
        ea.packed_plan(cu, **dict(dict(tokens=10), **kw))


def test_packed_abi():
    n = ctypes.c_size_t()
    lib = ea._lib
    assert lib.entmax_packed_plan_bytes(100, 3, ctypes.byref(n)) == ea.EA_OK and n.value > 0
    assert lib.entmax_packed_plan_bytes(0, 3, ctypes.byref(n)) == ea.EA_ERR_INVALID_ARG
    assert lib.entmax_packed_plan_bytes(100, 0, ctypes.byref(n)) == ea.EA_ERR_INVALID_ARG
    assert lib.entmax_packed_plan_bytes(100, 3, None) == ea.EA_ERR_INVALID_ARG
    assert lib.entmax_packed_plan_bytes(2 ** 31 - 1, 2 ** 31 - 1, ctypes.byref(n)) == ea.EA_ERR_UNSUPPORTED
    p, z = ea.default_params(), ea.PackedSizes()
    good = (100, 3, 50, 8, 2, 64, ea.EA_BF16)
    sizes = lambda s: lib.entmax_packed_sizes(ctypes.byref(ea.PackedShape(*s)), ctypes.byref(p), ctypes.byref(z))
    assert sizes(good) == ea.EA_OK
    for at, value, code in ((2, 0, 1), (2, 131073, 2), (3, 7, 1), (3, 0, 1), (4, 0, 1), (5, 80, 2), (6, 2, 2),
                            (0, -4, 1)):
        bad = list(good)
        bad[at] = value
        assert sizes(bad) == code, (at, value)
    # null pointers and small buffers, all before a launch
    s = ea.PackedShape(*good)
    st = ea.PackedStrides(*[ea.Strides(512, 64)] * 4)
    assert sizes(good) == ea.EA_OK
    call = lambda plan_, res_bytes, strides: lib.entmax_packed_fwd(
        ctypes.byref(s), ctypes.byref(p), plan_, 4096, 4096, 4096, 4096, strides, 0, 4096, res_bytes, None, 0, None, 0, None)
    assert call(None, z.residuals, st) == ea.EA_ERR_INVALID_ARG
    assert call(4096, z.residuals - 1, st) == ea.EA_ERR_WORKSPACE
    assert call(4096, z.residuals, ea.PackedStrides(*[ea.Strides(511, 64)] * 4)) == ea.EA_ERR_INVALID_ARG
    assert call(4096, z.residuals, ea.PackedStrides(*[ea.Strides(-512, 64)] * 4)) == ea.EA_ERR_INVALID_ARG
    assert call(4096, z.residuals, ea.PackedStrides(*[ea.Strides(1 << 25, 64)] * 4)) == ea.EA_ERR_INVALID_ARG


def decode_args(**kw):
    a = dict(q=torch.zeros(3, 4, 64, dtype=BF), k_cache=torch.zeros(3, 7, 2, 64, dtype=BF),
             v_cache=torch.zeros(3, 7, 2, 64, dtype=BF), lengths=torch.zeros(3, dtype=torch.int32))
    a.update(kw)
    return a


@pytest.mark.parametrize("change,word", [
    (dict(q=torch.zeros(3, 4, 64, dtype=torch.float16)), "bfloat16"),
    (dict(k_cache=torch.zeros(3, 7, 3, 64, dtype=BF)), "multiple"),
    (dict(v_cache=torch.zeros(3, 8, 2, 64, dtype=BF)), "shape"),
    (dict(k_cache=torch.zeros(3, 7, 2, 64)), "dtype"),
    (dict(lengths=torch.zeros(3, dtype=torch.int64)), "dtype"),
    (dict(lengths=torch.zeros(4, dtype=torch.int32)), "shape"),
    (dict(k_prefix=torch.zeros(9, 2, 64, dtype=BF)), "together"),
    (dict(k_prefix=torch.zeros(9, 4, 64, dtype=BF), v_prefix=torch.zeros(9, 4, 64, dtype=BF)), "shape"),
    (dict(out=torch.zeros(3, 4, 64)), "dtype"),
    (dict(workspace=torch.zeros(16, dtype=torch.uint8)), "workspace"),
    (dict(), "GPU"),
])
def test_prefix_decode_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        ea.prefix_decode(**decode_args(**change))


def test_prefix_decode_refuses_overlap():
    a = decode_args()
    with pytest.raises(ValueError, match="overlaps q"):
        ea.prefix_decode(**dict(a, out=a["q"]))


@pytest.mark.parametrize("at,value,code", [(0, -1, 1), (1, 3, 1), (2, 0, 1), (3, 32, 2), (4, 9, 2), (5, -1, 1),
                                           (5, 131072, 2), (6, -2, 1)])
def test_prefix_decode_abi(at, value, code):
    good, n = [3, 4, 2, 64, ea.EA_BF16, 100, 7], ctypes.c_size_t()
    assert ea._lib.entmax_prefix_decode_workspace(ctypes.byref(ea.DecodeShape(*good)), ctypes.byref(n)) == ea.EA_OK
    assert n.value >= 3 * 4 * 107 * 4
    good[at] = value
    assert ea._lib.entmax_prefix_decode_workspace(ctypes.byref(ea.DecodeShape(*good)), ctypes.byref(n)) == code


def test_rows_too_far_apart():
    """A tile's offsets are 32-bit numbers: refused by the binding, and by the C entry points."""
    far = (1 << 24) + 8
    for i in range(4):
        rows = [64] * 8
        rows[2 * i] = far
        with pytest.raises(ValueError, match="apart"):
            ea._packed_strides_of(*rows)
    for i in (4, 8):
        rows = [64] * 14
        rows[i] = far
        with pytest.raises(ValueError, match="apart"):
            ea._decode_strides_of(*rows)
    shape = ea.DecodeShape(1, 1, 1, 64, ea.EA_BF16, 64, 64)
    params = ea.make_params(1.5, None, False, False, None, 1e-6, head_dim=64)
    near, far = ea.Strides(64, 64), ea.Strides(far, 64)
    for k, kp in ((far, near), (near, far)):
        strides = ea.DecodeStrides(near, near, k, near, kp, near, 4096, 4096)
        assert ea._lib.entmax_prefix_decode(shape, params, strides, 4096, 4096, 4096, 4096, 4096, 4096, 4096, 4096,
                                            1 << 20, None) == ea.EA_ERR_INVALID_ARG


def test_grids_of_one_launch():
    """What a launch cannot hold is refused by the sizes, before any launch."""
    lib, n, sizes = ea._lib, ctypes.c_size_t(), ea.PackedSizes()
    params = ea.make_params(1.5, None, True, True, None, None, head_dim=64)
    size = lambda tokens, heads: lib.entmax_packed_sizes(ea.PackedShape(tokens, 1, 1000, heads, 1, 64, ea.EA_BF16),
                                                        ctypes.byref(params), ctypes.byref(sizes))
    assert size(64 * (2 ** 20 - 2), 4) == ea.EA_OK
    assert size(64 * (2 ** 20 - 1), 4) == ea.EA_ERR_UNSUPPORTED
    rows = lambda requests: lib.entmax_prefix_decode_workspace(
        ea.DecodeShape(requests, 8, 1, 64, ea.EA_BF16, 64, 64), ctypes.byref(n))
    assert rows(2 ** 20 - 1) == ea.EA_OK
    assert rows(2 ** 20) == ea.EA_ERR_UNSUPPORTED
    tokens = lambda t: lib.entmax_norm_rotary_workspace(
        ea.Rotary(t, 1, 1, 64, ea.EA_BF16, ea.EA_BF16, 64, 0, 1, (ctypes.c_int32 * 4)(32), 1e-6), ctypes.byref(n))
    assert tokens(2 ** 25) == ea.EA_OK
    assert tokens(2 ** 25 + 1) == ea.EA_ERR_UNSUPPORTED
