"""What calls over chunks write lies apart from the cache that they read or write: refused before anything is enqueued, on the
stage's own pool, from its first byte to its last.  CPU only: addresses are numbers, and no call here reaches a launch."""
import ctypes as C

import pytest

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk

DESC = cdb.make_desc(cdbgen.TINY)
ROWS, PAGES, POOL = 8, 4, 1 << 30
D = DESC.d
LAYERS = (DESC.n_prelude, DESC.n_core, DESC.n_coda)


def pool_bytes(stage):
    return LAYERS[stage] * PAGES * 2 * D * DESC.page_tokens * 2


def kv(stage):
    """The stage's pool at POOL, the others elsewhere."""
    at = [(5 + i) << 32 for i in range(3)]
    at[stage] = POOL
    return cdb.cdb_kv(*at, PAGES, PAGES, PAGES, 16, 4, 8)


CHUNKS = chunk.cdb_chunks(2, ROWS, 16, 16, 16, 16)


def qkv_call(stage, q_out, q=1 << 20, k=2 << 20, v=3 << 20):
    x = chunk.cdb_qkv(q, k, v, chunk.CDB_BF16, 0, D, D, D, None, None, None)
    return chunk.lib().cdb_chunk_qkv(C.byref(DESC), C.byref(kv(stage)), C.byref(CHUNKS), stage, 0, C.byref(x), q_out, chunk.CDB_BF16,
                                     16, 1 << 40, None)


def attend(stage, out):
    return chunk.lib().cdb_chunk_attention(C.byref(DESC), C.byref(kv(stage)), C.byref(CHUNKS), stage, 0, 1 << 20, chunk.CDB_BF16, out,
                                           chunk.CDB_ORDER_ROWS, 16, 1 << 40, None)


@pytest.mark.parametrize("stage", [0, 1, 2])
def test_the_cache_is_no_buffer_of_a_call(stage):
    n = ROWS * D * 2
    inside = (POOL, POOL + 16, POOL - n + 16, POOL + pool_bytes(stage) - 16, POOL + pool_bytes(stage) - n)
    for at in inside:
        assert attend(stage, at) == cdb.CDB_ERR_INVALID_ARG, at
        assert qkv_call(stage, at) == cdb.CDB_ERR_INVALID_ARG, at
        for part in ("q", "k", "v"):
            assert qkv_call(stage, 16 << 20, **{part: at}) == cdb.CDB_ERR_INVALID_ARG, (part, at)
