"""A cache in pages and in 4 bits, without a GPU: where its tokens lie and what its
tables say, in a build of the library's own header for the host; and refusals."""
import ctypes
import os
import random
import subprocess

import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")
from tests import pages_util  # noqa: E402

BF, I32 = torch.bfloat16, torch.int32
CSRC = os.path.join(os.path.dirname(ea.LIB_PATH), "csrc")
SHIM = r"""
#include "ea_pages.h"
using namespace ea;
extern "C" {
int32_t t_page_of(int32_t pages, int32_t shift, const int32_t* ids, int32_t rows, int32_t width, int64_t stride,
                  int32_t row, int32_t at) {
  return page_of(PageDims{pages, shift, 1, 64}, PageTable{ids, rows, width, stride}, row, at);
}
int64_t t_tile_at(int32_t pages, int32_t shift, int32_t heads, int32_t d, int32_t page, int32_t head, int32_t values,
                  int32_t at) {
  return tile_at(PageDims{pages, shift, heads, d}, page, head, values != 0, at);
}
int64_t t_page_bytes(int32_t shift, int32_t heads, int32_t d) { return page_bytes(PageDims{1, shift, heads, d}); }
void t_plan_row(int32_t length, int32_t count, int32_t width, int32_t shift, int32_t* out) {
  const RowPlan r = plan_row(length, count, width, shift);
  out[0] = r.old; out[1] = r.wanted; out[2] = r.kept; out[3] = r.grown; out[4] = r.fits; out[5] = r.writes;
}
int32_t t_copies(int32_t holders, int32_t writers, int32_t lowest, int32_t row) {
  return copies(holders, writers, lowest, row);
}
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    d = tmp_path_factory.mktemp("pages")
    (d / "shim.cpp").write_text(SHIM)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "shim.so"),
                           str(d / "shim.cpp")])
    lib = ctypes.CDLL(str(d / "shim.so"))
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    lib.t_page_of.argtypes = [i32, i32, ctypes.c_void_p, i32, i32, i64, i32, i32]
    lib.t_tile_at.restype = lib.t_page_bytes.restype = i64
    return lib


def test_page_of(host):
    ids = torch.tensor([[3, 0, -1, 9], [10, -2147483648, 2147483647, 1]], dtype=I32)
    def page(row, at):
        return host.t_page_of(10, 5, ids.data_ptr(), 2, 4, 4, row, at)
    assert [page(0, 32 * i) for i in range(4)] == [3, 0, -1, 9]
    assert [page(1, 32 * i + 31) for i in range(4)] == [-1, -1, -1, 1]  # numbers of no page
    big = 2 ** 31 - 1
    for row, at in ((-1, 0), (2, 0), (big, 0), (-big, 0), (0, -1), (0, 128), (0, big), (0, -big - 1), (2, big)):
        assert page(row, at) == -1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shift", [4, 5, 10])
def test_tiles_cover_the_cache_once(host, d, shift):
    pages, heads, tile = 3, 5, 17 * d // 2
    assert host.t_page_bytes(shift, heads, d) == heads * 2 * (1 << shift) // 16 * tile
    seen = sorted(host.t_tile_at(pages, shift, heads, d, p, h, v, at + 7)
                  for p in range(pages) for h in range(heads) for v in (0, 1) for at in range(0, 1 << shift, 16))
    assert seen == [tile * i for i in range(len(seen))] and len(seen) * tile == pages * host.t_page_bytes(shift, heads, d)
    # the tensor's order: [pages, kv_heads, 2, tiles, bytes]; a token behind the first page is in its own page's tile
    assert host.t_tile_at(pages, shift, heads, d, 1, 2, 1, (1 << shift) * 6) == tile * (((1 * heads + 2) * 2 + 1) << (shift - 4))
    # a pool of more than 2^32 bytes
    assert host.t_tile_at(1 << 20, shift, heads, d, (1 << 20) - 1, 4, 1, 0) == \
        ((1 << 20) - 1) * host.t_page_bytes(shift, heads, d) + 9 * (tile << (shift - 4))


def test_plan_row(host):
    out = (ctypes.c_int32 * 6)()
    rng = random.Random(3)
    edge = [0, 1, 15, 16, 17, 31, 32, 33, 64, 79, 80, 81, -1, 2 ** 31 - 1, -2 ** 31]
    for length in edge + [rng.randrange(90) for _ in range(30)]:
        for count in edge + [rng.randrange(-90, 90) for _ in range(30)]:
            host.t_plan_row(length, count, 5, 4, out)
            old, wanted, kept, grown, fits, writes = list(out)
            table = [[100 + i for i in range(5)]]
            new, lengths, missing, _ = pages_util.update_by_hand(table, [length], [0], [count], 16, 200)
            assert (fits, wanted) == (missing[0] != -1, lengths[0])
            assert new[0][:kept] == table[0][:kept] and kept + grown == sum(p >= 0 for p in new[0])
            assert new[0][kept:kept + grown] == list(range(grown))  # (free pages, lowest first)
            assert old == min(max(length, 0), 80)
            assert writes == (wanted > old and old % 16 != 0)


def test_copies(host):
    # alone; all holders write: the lowest keeps it; one holder does not write: every writer gets a copy
    assert host.t_copies(1, 1, 4, 4) == 0
    assert [host.t_copies(3, 3, 4, r) for r in (4, 5, 6)] == [0, 1, 1]
    assert [host.t_copies(3, 2, 4, r) for r in (4, 6)] == [1, 1]


def test_format_by_hand():
    x = torch.zeros(4, 32, dtype=torch.float64)
    x[0, :12] = torch.tensor([7.0, 5.0, -5.1, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, -0.0, -6.0])
    x[1, 0] = 7.0001  # the next scale: 4
    x[2, 1] = 3e38
    x[3, 5] = float("inf")
    code, scale = pages_util.pack(x)
    assert scale[:, 0].tolist() == [127, 128, 252, 255]
    assert code[0, :12].tolist() == [7, 6, 15, 0, 1, 2, 2, 4, 4, 6, 8, 15]
    assert code[1, 0] == 6 and code[2, 1] == 7
    v = pages_util.unpack(code, scale)
    assert v[0, 0] == 6 and v[1, 0] == 8 and torch.isnan(v[3]).all()
    assert v[2, 1] == 6 * 2.0 ** 125


# ---------------------------------------------------------------- refusals

def cache(pages=6, page=16, hk=2, d=64, layers=None):
    return torch.zeros(((layers,) if layers else ()) + (pages, hk, 2, page // 16, 17 * d // 2), dtype=torch.uint8)


def ints(*v):
    return torch.tensor(v, dtype=I32)


def rows_args(**kw):
    a = dict(cache=cache(), k=torch.zeros(3, 2, 64, dtype=BF), v=torch.zeros(3, 2, 64, dtype=BF), rows=ints(0, 1, 1),
             positions=ints(0, 0, 1), table=torch.zeros(2, 4, dtype=I32))
    a.update(kw)
    return a


@pytest.mark.parametrize("change,word", [
    (dict(cache=cache().int()), "uint8"),
    (dict(cache=cache(layers=2)), "layer"),
    (dict(cache=cache()[..., :-1]), "17 head_dim"),
    (dict(cache=cache(pages=12)[::2]), "contiguous"),
    (dict(cache=torch.zeros(6 * 2 * 2 * 544 + 8, dtype=torch.uint8)[8:].view(6, 2, 2, 1, 544)), "16 bytes"),
    (dict(cache=torch.zeros(6, 2, 3, 1, 544, dtype=torch.uint8)), "layer's cache"),
    (dict(table=torch.zeros(2, 4, dtype=torch.int64)), "table"),
    (dict(table=torch.zeros(4, dtype=I32)), "table"),
    (dict(table=torch.zeros(2, 0, dtype=I32)), "entries"),
    (dict(table=torch.zeros(4, 2, dtype=I32).t()), "contiguous"),
    (dict(table=torch.zeros(2, 8193, dtype=I32)), "131072"),
    (dict(rows=ints(0, 1)), "positions"),
    (dict(rows=torch.zeros(3, dtype=torch.int64)), "rows"),
    (dict(positions=torch.zeros(3, dtype=torch.int64)), "positions"),
    (dict(k=torch.zeros(3, 2, 64, dtype=torch.float16)), "bfloat16"),
    (dict(k=torch.zeros(4, 2, 64, dtype=BF)), "shape"),
    (dict(k=torch.zeros(3, 1, 64, dtype=BF)), "shape"),
    (dict(v=torch.zeros(3, 2, 64)), "dtype"),
    (dict(v=torch.zeros(3, 64, 2, dtype=BF).transpose(1, 2)), "contiguous"),
    (dict(k=torch.zeros(3, 2, 68, dtype=BF)[..., :64]), "16 bytes"),
    (dict(), "GPU"),
])
def test_append_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        ea.cache_append(**rows_args(**change))


@pytest.mark.parametrize("page", [8, 24, 48, 2048])
def test_page_sizes(page):
    with pytest.raises((ValueError, ea.EntmaxAttnError)):
        ea.paged_cache(4, page, 2, 64, device="cpu")


def test_read_refuses():
    a = rows_args()
    del a["k"], a["v"]
    base = torch.zeros(4, 2, 64, dtype=BF)
    for change, word in ((dict(dtype=torch.float16), "dtype"), (dict(k_out=torch.zeros(3, 2, 64)), "dtype"),
                         (dict(k_out=base[:3], v_out=base[1:]), "overlaps"),
                         (dict(v_out=torch.zeros(3, 1, 64, dtype=BF).expand(3, 2, 64)), "memory|16 bytes"), (dict(), "GPU")):
        with pytest.raises(ValueError, match=word):
            ea.cache_read(**dict(a, **change))


def update_args(**kw):
    a = dict(cache=cache(layers=2), table=torch.zeros(2, 4, dtype=I32), lengths=ints(5, 3), parents=ints(0, 0, 1),
             counts=ints(1, 1, 0))
    a.update(kw)
    return a


def test_update_refuses():
    t, i = torch.zeros(3, 4, dtype=I32), ints(0, 0, 0)
    out = dict(table_out=t, lengths_out=i, missing_out=i.clone())
    a = update_args()
    wide = torch.zeros(3, 8, dtype=I32)
    for change, word in (
            (dict(lengths=ints(5)), "lengths"), (dict(parents=torch.zeros(3, dtype=torch.int64)), "parents"),
            (dict(counts=ints(1)), "counts"), (dict(table_out=t), "together"),
            (dict(out, table_out=torch.zeros(3, 5, dtype=I32)), "table_out must be"), (dict(out, lengths_out=ints(1)), "lengths_out"),
            (dict(out, missing_out=i), "overlaps"), (dict(out, table=t, lengths=i.clone()), "overlaps table"),
            (dict(out, parents=i), "overlaps parents"), (dict(out, table_out=t[:1].expand(3, 4)), "memory"),
            (dict(out, table=wide[:, :4], lengths=i.clone(), table_out=wide[:, 4:]), "overlaps|GPU"),
            (dict(workspace=torch.zeros(8, dtype=torch.uint8)), "workspace"),
            (dict(cache=cache(layers=2)[:, ::2]), "contiguous"), (dict(), "GPU")):
        with pytest.raises(ValueError, match=word):
            ea.cache_update(**dict(a, **change))


def test_compact_refuses():
    a = dict(cache=cache(layers=2), table=torch.zeros(2, 4, dtype=I32), lengths=ints(5, 3))
    t = torch.zeros(2, 4, dtype=I32)
    for change, word in ((dict(lengths=ints(5)), "lengths"), (dict(table_out=t), "together"),
                         (dict(table_out=t, used_out=ints(1, 2)), "used_out"),
                         (dict(table_out=a["table"], used_out=ints(1)), "overlaps"),
                         (dict(table_out=t[:1], used_out=ints(1)), "table_out must be"), (dict(), "GPU")):
        with pytest.raises(ValueError, match=word):
            ea.cache_compact(**dict(a, **change))


def decode_args(**kw):
    a = dict(q=torch.zeros(2, 4, 64, dtype=BF), cache=cache(), table=torch.zeros(2, 4, dtype=I32), lengths=ints(5, 3))
    a.update(kw)
    return a


@pytest.mark.parametrize("change,word", [
    (dict(q=torch.zeros(2, 4, 128, dtype=BF)), "head_dim"),
    (dict(q=torch.zeros(2, 3, 64, dtype=BF)), "multiple"),
    (dict(q=torch.zeros(2, 0, 64, dtype=BF)), "multiple"),
    (dict(q=torch.zeros(2, 4, 64, dtype=torch.float16)), "bfloat16"),
    (dict(q=torch.zeros(2, 256, dtype=BF)), "heads"),
    (dict(q=torch.zeros(3, 4, 64, dtype=BF), lengths=ints(1, 2, 3)), "give rows"),
    (dict(lengths=ints(5)), "lengths"),
    (dict(rows=ints(0)), "rows"),
    (dict(rows=torch.zeros(2, dtype=torch.int64)), "rows"),
    (dict(out=torch.zeros(2, 4, 64)), "dtype"),
    (dict(workspace=torch.zeros(16, dtype=torch.uint8)), "workspace"),
    (dict(), "GPU"),
])
def test_decode_refuses(change, word):
    with pytest.raises(ValueError, match=word):
        ea.paged_decode(**decode_args(**change))
    q = torch.zeros(2, 4, 64, dtype=BF)
    with pytest.raises(ValueError, match="overlaps"):
        ea.paged_decode(**decode_args(q=q, out=q))


ADDRESS = 1 << 20  # (of nothing: these calls end before they look)


def c_table(width=4, rows=2, stride=4):
    return ea.PageTable(rows, width, stride)


@pytest.mark.parametrize("c,code", [
    (ea.Cache(0, 16, 2, 64), ea.EA_ERR_INVALID_ARG), (ea.Cache(4, 16, 0, 64), ea.EA_ERR_INVALID_ARG),
    (ea.Cache(4, 0, 2, 64), ea.EA_ERR_INVALID_ARG), (ea.Cache(4, 8, 2, 64), ea.EA_ERR_UNSUPPORTED),
    (ea.Cache(4, 24, 2, 64), ea.EA_ERR_UNSUPPORTED), (ea.Cache(4, 2048, 2, 64), ea.EA_ERR_UNSUPPORTED),
    (ea.Cache(4, 16, 2, 96), ea.EA_ERR_UNSUPPORTED), (ea.Cache(1 << 21, 1024, 2, 64), ea.EA_ERR_UNSUPPORTED),
    (ea.Cache(4, 16, 1 << 17, 64), ea.EA_ERR_UNSUPPORTED)])
def test_cache_abi(c, code):
    n = ctypes.c_size_t()
    assert ea._lib.entmax_cache_page_bytes(c, ctypes.byref(n)) == code
    assert ea._lib.entmax_cache_workspace(c, 1, ctypes.byref(n)) == code
    assert ea._lib.entmax_paged_decode_workspace(ea.PagedShape(1, 2, 0, 8), c, ctypes.byref(n)) == code
    s = ea.Strides(128, 64)
    assert ea._lib.entmax_cache_append(c, ADDRESS, c_table(), ADDRESS, 1, 0, ADDRESS, ADDRESS, ADDRESS, s, ADDRESS, s, None) == code


OK_CACHE = ea.Cache(4, 16, 2, 64)


@pytest.mark.parametrize("change,code", [
    (dict(table=c_table(width=0)), ea.EA_ERR_INVALID_ARG), (dict(table=c_table(rows=0)), ea.EA_ERR_INVALID_ARG),
    (dict(table=c_table(stride=-4)), ea.EA_ERR_INVALID_ARG), (dict(ids=None), ea.EA_ERR_INVALID_ARG),
    (dict(ids=ADDRESS + 2), ea.EA_ERR_INVALID_ARG),
    (dict(table=c_table(width=8193, stride=8193)), ea.EA_ERR_UNSUPPORTED),
    (dict(tokens=-1), ea.EA_ERR_INVALID_ARG), (dict(tokens=1 << 26), ea.EA_ERR_UNSUPPORTED),
    (dict(dtype=2), ea.EA_ERR_UNSUPPORTED), (dict(k=ADDRESS + 8), ea.EA_ERR_INVALID_ARG), (dict(v=None), ea.EA_ERR_INVALID_ARG),
    (dict(rows=None), ea.EA_ERR_INVALID_ARG), (dict(positions=ADDRESS + 1), ea.EA_ERR_INVALID_ARG),
    (dict(cache=None), ea.EA_ERR_INVALID_ARG), (dict(ks=ea.Strides(127, 64)), ea.EA_ERR_INVALID_ARG),
    (dict(tokens=0), ea.EA_OK)])
def test_rows_abi(change, code):
    a = dict(cache=ADDRESS, table=c_table(), ids=ADDRESS, tokens=1, dtype=0, rows=ADDRESS, positions=ADDRESS, k=ADDRESS,
             ks=ea.Strides(128, 64), v=ADDRESS, vs=ea.Strides(128, 64))
    a.update(change)
    for f in (ea._lib.entmax_cache_append, ea._lib.entmax_cache_read):
        assert f(OK_CACHE, *a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(layers=0), ea.EA_ERR_INVALID_ARG), (dict(rows=-1), ea.EA_ERR_INVALID_ARG),
    (dict(rows=(1 << 20) + 1), ea.EA_ERR_UNSUPPORTED), (dict(out_stride=3), ea.EA_ERR_INVALID_ARG),
    (dict(lengths=None), ea.EA_ERR_INVALID_ARG), (dict(parents=None), ea.EA_ERR_INVALID_ARG),
    (dict(counts=ADDRESS + 2), ea.EA_ERR_INVALID_ARG), (dict(table_out=None), ea.EA_ERR_INVALID_ARG),
    (dict(lengths_out=None), ea.EA_ERR_INVALID_ARG), (dict(missing=None), ea.EA_ERR_INVALID_ARG),
    (dict(workspace=None), ea.EA_ERR_INVALID_ARG), (dict(nbytes=64), ea.EA_ERR_WORKSPACE), (dict(rows=0), ea.EA_OK)])
def test_update_abi(change, code):
    a = dict(layers=1, cache=ADDRESS, table=c_table(), ids=ADDRESS, lengths=ADDRESS, rows=3, parents=ADDRESS, counts=ADDRESS,
             table_out=ADDRESS, out_stride=4, lengths_out=ADDRESS, missing=ADDRESS, workspace=ADDRESS, nbytes=1 << 20)
    a.update(change)
    assert ea._lib.entmax_cache_update(OK_CACHE, *a.values(), None) == code


@pytest.mark.parametrize("change,code", [
    (dict(shape=ea.PagedShape(-1, 4, 0, 64)), ea.EA_ERR_INVALID_ARG), (dict(shape=ea.PagedShape(2, 3, 0, 64)), ea.EA_ERR_INVALID_ARG),
    (dict(shape=ea.PagedShape(2, 4, 2, 64)), ea.EA_ERR_UNSUPPORTED), (dict(shape=ea.PagedShape(2, 4, 0, -1)), ea.EA_ERR_INVALID_ARG),
    (dict(shape=ea.PagedShape(2, 4, 0, 131073)), ea.EA_ERR_UNSUPPORTED),
    (dict(shape=ea.PagedShape(1 << 21, 4, 0, 64)), ea.EA_ERR_UNSUPPORTED),
    (dict(shape=ea.PagedShape(1 << 18, 4, 0, 65536)), ea.EA_ERR_UNSUPPORTED),
    (dict(alpha=2.01), ea.EA_ERR_UNSUPPORTED), (dict(alpha=1.0), ea.EA_ERR_INVALID_ARG),
    (dict(q=None), ea.EA_ERR_INVALID_ARG), (dict(lengths=None), ea.EA_ERR_INVALID_ARG), (dict(rows=ADDRESS + 1), ea.EA_ERR_INVALID_ARG),
    (dict(o=ADDRESS + 4), ea.EA_ERR_INVALID_ARG), (dict(workspace=None), ea.EA_ERR_INVALID_ARG),
    (dict(nbytes=1000), ea.EA_ERR_WORKSPACE), (dict(shape=ea.PagedShape(0, 4, 0, 64)), ea.EA_OK)])
def test_decode_abi(change, code):
    a = dict(shape=ea.PagedShape(2, 4, 0, 64), alpha=1.5, cache=ADDRESS, table=c_table(), ids=ADDRESS, q=ADDRESS, qs=ea.Strides(256, 64),
             lengths=ADDRESS, rows=None, o=ADDRESS, os=ea.Strides(256, 64), workspace=ADDRESS, nbytes=1 << 24)
    a.update(change)
    p = ea.make_params(a.pop("alpha"))
    shape = a.pop("shape")
    assert ea._lib.entmax_paged_decode(shape, p, OK_CACHE, *a.values(), None) == code


def test_workspace_counts():
    q = torch.zeros(3, 4, 64, dtype=BF)
    c = cache()
    t = torch.zeros(3, 200, dtype=I32)  # 3200 tokens: 4 regions
    assert ea.paged_decode_workspace(q, c, t) >= 3 * 4 * 4 * 1024 * 8
    assert ea.paged_decode_workspace(q, c, t, max_length=1000) < ea.paged_decode_workspace(q, c, t)
    assert ea.paged_decode_workspace(q, c, t, max_length=0) == 0
    assert ea.cache_workspace(cache(layers=3), 7) > 0
