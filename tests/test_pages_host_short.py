"""Updates of page tables with too few pages, without a GPU: no row loses a token."""
import ctypes
import os
import random
import subprocess

import pytest

torch = pytest.importorskip("torch")
ea = pytest.importorskip("paper_2502_12082_amd", reason="HIP library not built")
from tests import pages_rules as pr  # noqa: E402

CSRC = os.path.join(os.path.dirname(ea.LIB_PATH), "csrc")


def test_no_token_is_lost_by_the_rule():
    """(The rule by which one row keeps a page that all of its holders write to.)"""
    short = 0
    for seed in range(400):
        page, pages, width, step, steps = pr.short_steps(seed)
        pool = pr.Pool(page, pages, width)
        for _ in range(steps):
            parents, counts = step(len(pool.rows))
            table, lengths, missing, copies = pr.update_by_rule(pool.table, pool.lengths(), parents, counts, page, pages)
            new = pool.step(parents, counts, table, lengths, missing)
            pool.write(copies, new)
            assert pool.lost() == [], (seed, parents, counts)
            short += any(m > 0 for m in missing)
    assert short > 1000


def test_keeper(tmp_path):
    """The library's number of a writing row: the smallest is of the row furthest into the page, ties of the lowest."""
    (tmp_path / "shim.cpp").write_text(r"""
#include "ea_pages.h"
extern "C" int32_t t_keeper_key(int32_t old, int32_t shift, int32_t row) { return ea::keeper_key(old, shift, row); }
extern "C" int32_t t_keeper_row(int32_t key) { return ea::keeper_row(key); }
""")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(tmp_path / "shim.so"),
                           str(tmp_path / "shim.cpp")])
    lib = ctypes.CDLL(str(tmp_path / "shim.so"))
    rng = random.Random(1)
    for shift in (4, 7, 10):
        page = 1 << shift
        rows = [(rng.choice([rng.randrange(1 << 17), page - 1, 1, page + 1, 131071]), rng.choice([0, 1, 255, (1 << 20) - 1, rng.randrange(1 << 20)]))
                for _ in range(200)]
        keys = {(old, row): lib.t_keeper_key(old, shift, row) for old, row in rows}
        for (old, row), key in keys.items():
            assert 0 <= key < 2 ** 31 - 1 and lib.t_keeper_row(key) == row
        order = sorted(keys, key=lambda x: keys[x])
        assert [(-(old % page), row) for old, row in order] == sorted((-(old % page), row) for old, row in keys)
