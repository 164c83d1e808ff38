"""GPU: calls over chunks with page tables of the largest size, at the last positions that those have, and with buffers of
many more rows than chunks."""
import numpy as np
import pytest
import torch

import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk
from test_gpu_chunk import PAGE, Case, Write, _dev, _say

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


def test_rows_outside_chunks_are_not_read():
    """65536 rows of three parts, 16 x 128 values of 4 bytes each, are 1.6 GB: 0.2 ms at the 8 TB/s that this memory cannot
    exceed.  A call in which chunks have 13 of the rows takes less than 0.6 of that, from its first rows to its last."""
    _say("rows that nobody has")
    H, hd, n, M = 16, 128, 13, 65536
    c = Case(H, hd, [(n, 40, 0, 0)], seed=63).device()
    x = torch.randn((M, 3, H, hd), device="cuda")
    qkv = chunk.QKV(*x.unbind(1), norm=True)
    q_out = torch.zeros((M, H * hd), device="cuda")
    for first in (0, 1000, M - n):
        c.c = chunk.Chunks(M, _dev([first, first + n]), c.c.seq, c.c.pos0, c.c.cc)
        q_out.fill_(77.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(4):
                chunk.cdb_chunk_qkv(c.desc, c.kv, c.c.c, 1, 1, qkv.c, q_out, c.ws.buf)
        took = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            graph.replay()
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b) / 4)
        assert c.code() == 0
        assert (q_out[first:first + n] != 77).all()
        assert (q_out[:first] == 77).all() and (q_out[first + n:] == 77).all()
        assert min(took) < 0.6 * x.numel() * 4 / 8e12 * 1e3, took
