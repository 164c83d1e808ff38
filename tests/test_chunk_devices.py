"""Tensors of another device than the workspace's are refused by the calls over chunks and by sampled acceptance, and holders
refuse tensors of two devices.  CPU only: the tensors are stand-ins, and no call here reaches the library."""
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk, tree

DESC = cdb.make_desc(cdbgen.TINY)
KV = cdb.cdb_kv(16, 16, 16, 1, 1, 1, 16, 4, 8)


class OnDevice:
    """What the binding looks at in a tensor, of a GPU that is not there."""

    def __init__(self, dtype, n, index=0):
        self.dtype, self.n, self.is_cuda, self.index = dtype, n, True, index

    def get_device(self):
        return self.index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def held(c, index):
    c.device = index
    return c


def chunks(index=0):
    return held(chunk.cdb_chunks(1, 4, 16, 16, 16, 16), index)


def qkv(index=0):
    return held(chunk.cdb_qkv(16, 16, 16, 1, 0, DESC.d, DESC.d, DESC.d, None, None, None), index)


def rows(index=0, dtype=torch.bfloat16):
    return OnDevice(dtype, 4 * DESC.d, index)


WS = OnDevice(torch.uint8, 1 << 20)
DRAFTS = lambda index=0: held(tree.cdb_drafts(2, 4, 2, None, None, 16, 16, 16), index)
SAMPLING = lambda index=0: held(tree.cdb_sampling(16, None, 1024, 0, None, None, 16, 16), index)
OUT = lambda index=0: held(tree.cdb_accepted(16, 16, 16), index)
IDS = lambda index=0: OnDevice(torch.int32, 2, index)
SAMPLED = (IDS, IDS, DRAFTS, SAMPLING, OUT)


def sampled(row0, first, drafts, sampling, out):
    return tree.cdb_tree_sample(DESC, drafts, row0, first, sampling, out, WS, n_rows=4)


CALLS = [lambda: chunk.cdb_chunk_qkv(DESC, KV, chunks(1), 1, 0, qkv(), rows(), WS),
         lambda: chunk.cdb_chunk_qkv(DESC, KV, chunks(), 1, 0, qkv(1), rows(), WS),
         lambda: chunk.cdb_chunk_qkv(DESC, KV, chunks(), 1, 0, qkv(), rows(1), WS),
         lambda: chunk.cdb_chunk_attention(DESC, KV, chunks(1), 1, 0, rows(), rows(), WS),
         lambda: chunk.cdb_chunk_attention(DESC, KV, chunks(), 1, 0, rows(1), rows(), WS),
         lambda: chunk.cdb_chunk_attention(DESC, KV, chunks(), 1, 0, rows(), rows(1), WS),
         *(lambda i=i: sampled(*(make(int(i == k)) for k, make in enumerate(SAMPLED))) for i in range(len(SAMPLED)))]


class Reached(Exception):
    pass


@pytest.fixture(autouse=True)
def no_library(monkeypatch):
    def stop(*_):
        raise Reached

    monkeypatch.setattr(tree, "_stream", stop)
    monkeypatch.setattr(chunk, "_stream", stop)


@pytest.mark.parametrize("i", range(len(CALLS)))
def test_another_device_is_refused(i):
    with pytest.raises(cdb.CdbError) as e:
        CALLS[i]()
    assert e.value.status == cdb.CDB_ERR_INVALID_ARG


def test_the_same_device_goes_on():
    for call in (lambda: chunk.cdb_chunk_qkv(DESC, KV, chunks(), 1, 0, qkv(), rows(), WS),
                 lambda: chunk.cdb_chunk_attention(DESC, KV, chunks(), 1, 0, rows(), rows(), WS),
                 lambda: sampled(*(make() for make in SAMPLED))):
        with pytest.raises(Reached):
            call()


def test_holders_of_two_devices():
    a, b = OnDevice(torch.int32, 2, 0), OnDevice(torch.int32, 2, 1)
    assert tree._held(chunk.cdb_chunks(), a, None, a).device == 0
    with pytest.raises(cdb.CdbError) as e:
        tree._held(chunk.cdb_chunks(), a, b)
    assert e.value.status == cdb.CDB_ERR_INVALID_ARG
