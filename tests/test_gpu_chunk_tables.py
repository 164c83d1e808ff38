"""GPU: calls over chunks with page tables of the largest size, and at the last positions that those have."""
import numpy as np
import pytest
import torch

import paper_2608_09444_amd as cdb
from test_gpu_chunk import PAGE, Case, Write, _say

pytestmark = pytest.mark.gpu

MOST_PAGES = (2 ** 31 - 1 - 64) // PAGE


def _widen(c, pages):
    """The case's table with as many pages per plane, those behind its own unmapped."""
    S, planes, P = c.table.shape
    wide = torch.full((S, planes, pages), -1, dtype=torch.int32, device="cuda")
    wide[:, :, :P] = c.d_table
    c.d_table = wide
    ptr = [None] * 3
    ptr[c.stage] = c.d_pool.data_ptr()
    count = [0] * 3
    count[c.stage] = c.pages
    c.kv = cdb.cdb_kv(*ptr, *count, wide.data_ptr(), S, pages)
    return c


@pytest.mark.parametrize("pages", [2 ** 26 + 1, 100_000_000, MOST_PAGES])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_short_contexts_in_wide_tables(dtype, pages):
    _say(f"wide table {dtype} {pages}")
    r = np.random.default_rng(61)
    for H, hd, chunks in ((4, 64, [(2100, 100, 0, 0)]), (2, 128, [(1, int(p), 0, 1) for p in r.integers(0, 900, 64)]),
                          (3, 96, [(13, 700, 0, 2)])):
        c = _widen(Case(H, hd, chunks, seed=61).device(), pages)
        got, q = c.attend(dtype)
        assert c.code() == 0
        c.check(got, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_last_positions_of_the_widest_table(dtype):
    """Five rows at the end, whose sequence has its last three pages only."""
    _say(f"last positions {dtype}")
    H, hd, n, pages = 4, 64, 5, 3
    c = Case(H, hd, [(n, pages * PAGE - n, 0, 1)], seed=62).device()
    ids = c.d_table[0, 2, :pages].clone()
    _widen(c, MOST_PAGES)
    c.d_table[0, 2, :pages] = -1
    c.d_table[0, 2, -pages:] = ids
    end = MOST_PAGES * PAGE
    c.c.pos0.fill_(end - n)
    got, q = c.attend(dtype)
    assert c.code() == cdb.CDB_DEV_UNMAPPED_PAGE
    c.check(got, q)  # as the same rows over the same pages at the beginning of a table
    w = Write(c, dtype, False, seed=62, rope=np.arange(n))
    w.run()
    assert c.code() == 0
    w.check()
