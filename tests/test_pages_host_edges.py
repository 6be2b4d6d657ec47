"""Calls on a cache in pages and in 4 bits that are refused, or are not, at the edge, without a GPU."""
import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")

I32 = torch.int32


def call(f, **kw):
    with pytest.raises(ValueError) as e:
        f(**kw)
    return str(e.value)


def test_columns_of_one_wider_table():
    """A table and the one to write may not be columns of the same rows: their ranges of memory meet.
    Behind each other in one buffer they are what is asked for (and end at the missing GPU)."""
    cache = torch.zeros(2, 6, 2, 2, 1, 544, dtype=torch.uint8)
    args = dict(cache=cache, lengths=torch.zeros(3, dtype=I32), parents=torch.zeros(3, dtype=I32), counts=torch.zeros(3, dtype=I32),
                lengths_out=torch.zeros(3, dtype=I32), missing_out=torch.zeros(3, dtype=I32))
    wide, rows = torch.zeros(3, 8, dtype=I32), torch.zeros(6, 4, dtype=I32)
    assert "table_out overlaps table" in call(ea.cache_update, table=wide[:, :4], table_out=wide[:, 4:], **args)
    assert "GPU" in call(ea.cache_update, table=rows[:3], table_out=rows[3:], **args)
    args = dict(cache=cache, lengths=torch.zeros(3, dtype=I32), used_out=torch.zeros(1, dtype=I32))
    assert "table_out overlaps table" in call(ea.cache_compact, table=wide[:, :4], table_out=wide[:, 4:], **args)
    assert "GPU" in call(ea.cache_compact, table=rows[:3], table_out=rows[3:], **args)


def test_sixteens_of_heads():
    """The bound of decoding's grid counts each 16 query heads of a key head."""
    import ctypes
    c, n = ea.Cache(4, 16, 2, 64), ctypes.c_size_t()
    for heads, queries, ok in ((32, 1 << 16, True), (32, 1 << 17, False), (34, 1 << 15, True), (34, 1 << 16, False)):
        status = ea._lib.entmax_paged_decode_workspace(ea.PagedShape(queries, heads, 0, 64 * 1024), c, ctypes.byref(n))
        assert status == (ea.EA_OK if ok else ea.EA_ERR_UNSUPPORTED), (heads, queries)
