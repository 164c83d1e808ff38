"""The Python binding of sampled acceptance over structs that are made by hand.  CPU only: a stand-in takes the C entry's
place."""
import types

import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree

DESC = cdb.make_desc(cdbgen.TINY)


class OnDevice:
    """What the binding looks at in a tensor, of a GPU that is not there."""

    def __init__(self, dtype, n, index=0):
        self.dtype, self.n, self.is_cuda, self.device = dtype, n, True, types.SimpleNamespace(index=index)

    def get_device(self):
        return self.device.index

    def numel(self):
        return self.n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def call(monkeypatch, sampling, **kw):
    """n_rows as the C entry gets it."""
    got = []

    class Entry:
        def cdb_tree_sample(self, *a):
            got.append(a[3])
            return cdb.CDB_OK

    monkeypatch.setattr(tree, "lib", Entry)
    monkeypatch.setattr(tree, "_stream", lambda fn, stream, ws: 0)
    ids = OnDevice(torch.int32, 2)
    drafts = tree.cdb_drafts(2, 4, 2, None, None, 16, 16, 16)
    tree.cdb_tree_sample(DESC, drafts, ids, ids, sampling, tree.cdb_accepted(16, 16, 16), OnDevice(torch.uint8, 1 << 20), **kw)
    return got[0]


def test_rows_of_a_struct_made_by_hand(monkeypatch):
    plain = tree.cdb_sampling(16, None, 1024, 0, None, None, 16, 16)
    assert call(monkeypatch, plain, n_rows=5) == 5
    with pytest.raises(cdb.CdbError) as e:
        call(monkeypatch, plain)
    assert e.value.status == cdb.CDB_ERR_INVALID_ARG


def test_rows_of_a_holder(monkeypatch):
    held = tree.cdb_sampling(16, None, 1024, 0, None, None, 16, 16)
    held.n_rows = 7
    assert call(monkeypatch, held) == 7
    assert call(monkeypatch, held, n_rows=3) == 3
    with pytest.raises(cdb.CdbError) as e:
        call(monkeypatch, held, n_rows=8)
    assert e.value.status == cdb.CDB_ERR_INVALID_ARG
