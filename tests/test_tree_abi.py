"""The C entries of include/libcdb_tree.h: exported, and bad arguments refused before anything is enqueued; the Python
holders refuse tensors that the kernels could not read.  CPU only (no call here reaches a launch)."""
import ctypes as C
import os
import re

import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DESC = cdb.make_desc(cdbgen.TINY)
BAD_DESC = cdb.make_desc(cdbgen.shrink(cdbgen.TINY, head_dim=80, n_heads=4, d=320))
BIG = 1 << 40
INVALID, CAPACITY, UNSUPPORTED = cdb.CDB_ERR_INVALID_ARG, cdb.CDB_ERR_CAPACITY, cdb.CDB_ERR_UNSUPPORTED


def _status(fn, *args):
    return getattr(tree.lib(), fn)(*(C.byref(a) if isinstance(a, C.Structure) else a for a in args))


def test_every_declared_entry_is_exported():
    text = open(os.path.join(ROOT, "include", "libcdb_tree.h")).read()
    names = re.findall(r"^(?:cdb_status|size_t)\s+(cdb_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(tree.EXPORTED)
    for n in names:
        assert hasattr(tree.lib(), n), n


@pytest.mark.parametrize("shape", [cdbgen.TINY, cdbgen.OURO, cdbgen.HUGINN], ids=lambda s: s.name)
def test_workspace_serves_every_smaller_call(shape):
    desc = cdb.make_desc(shape)
    sizes = [tree.cdb_tree_workspace_bytes(desc, r, 300) for r in range(cdb.MAX_ROWS + 1)]
    assert all(b >= a for a, b in zip(sizes, sizes[1:]))
    assert all(b >= cdb.cdb_workspace_bytes(desc, r) for r, b in enumerate(sizes))
    assert sizes[0] >= 256
    assert tree.cdb_tree_workspace_bytes(desc, cdb.MAX_ROWS + 1, 1) == 0
    assert tree.cdb_tree_workspace_bytes(desc, -1, 1) == 0
    assert tree.cdb_tree_workspace_bytes(desc, 1, -1) == 0
    assert tree.cdb_tree_workspace_bytes(BAD_DESC, 1, 1) == 0


def test_map_pages_refusals():
    one, two, three = (tree.cdb_page_pool(k, k, 8) for k in (1, 2, 3))

    def call(desc=DESC, table=1, S=2, P=4, pre=one, core=two, coda=three, layout=0, length=1, mapped=1, ws=1, nb=BIG):
        return _status("cdb_map_pages", desc, table, S, P, pre, core, coda, layout, length, mapped, ws, nb, None)

    for kw in ({"table": None}, {"length": None}, {"mapped": None}, {"ws": None}, {"layout": 3}, {"layout": -1}, {"S": -1},
               {"P": -1}, {"core": None}, {"pre": tree.cdb_page_pool(None, 1, 8)}, {"coda": tree.cdb_page_pool(1, None, 8)},
               {"core": tree.cdb_page_pool(2, 2, -1)}, {"core": one}, {"coda": tree.cdb_page_pool(2, 3, 8)},
               {"coda": tree.cdb_page_pool(3, 1, 8)}, {"desc": None}):
        assert call(**kw) == INVALID, kw
    assert call(desc=BAD_DESC) == UNSUPPORTED
    assert call(nb=255) == CAPACITY
    assert call(P=1 << 28) == CAPACITY
    assert call(S=1 << 20, P=1 << 20) == CAPACITY


def _drafts(**kw):
    a = dict(n_trees=2, max_nodes=8, max_seqs=4, seq=1, len=1, n_nodes=1, parent=1, tokens=1)
    a.update(kw)
    return tree.cdb_drafts(*a.values())


@pytest.mark.parametrize("kw,want", [({"n_trees": -1}, INVALID), ({"max_nodes": 0}, INVALID), ({"max_nodes": 65}, INVALID),
                                     ({"max_seqs": -1}, INVALID), ({"n_trees": 257}, CAPACITY)])
def test_bad_drafts_are_refused_alike(kw, want):
    d, acc = _drafts(**kw), tree.cdb_accepted(1, 1, 1)
    kv = cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 1, 1)
    assert _status("cdb_tree_rows", d, tree.cdb_row_map(8, *[1] * 8), 1, BIG, None) == want
    assert _status("cdb_tree_accept", d, 1, 1, 8, 1, acc, 1, BIG, None) == want
    assert _status("cdb_tree_commit", DESC, kv, d, acc, 1, BIG, None) == want


def test_tree_rows_refusals():
    def call(d=_drafts(), out=tree.cdb_row_map(8, *[1] * 8), ws=1, nb=BIG):
        return _status("cdb_tree_rows", d, out, ws, nb, None)

    for f in ("seq", "len", "n_nodes", "parent", "tokens"):
        assert call(d=_drafts(**{f: None})) == INVALID, f
    for i in range(8):
        assert call(out=tree.cdb_row_map(8, *[None if k == i else 1 for k in range(8)])) == INVALID, i
    assert call(out=tree.cdb_row_map(-1, *[1] * 8)) == INVALID
    assert call(out=None) == INVALID
    assert call(ws=None) == INVALID
    assert call(nb=255) == CAPACITY


def test_tree_accept_refusals():
    def call(d=_drafts(seq=None, len=None), row0=1, ids=1, n=8, first=1, out=tree.cdb_accepted(1, 1, 1), ws=1, nb=BIG):
        return _status("cdb_tree_accept", d, row0, ids, n, first, out, ws, nb, None)

    for kw in ({"row0": None}, {"ids": None}, {"first": None}, {"out": None}, {"ws": None}, {"n": -1},
               {"out": tree.cdb_accepted(None, 1, 1)}, {"out": tree.cdb_accepted(1, None, 1)},
               {"out": tree.cdb_accepted(1, 1, None)}, {"d": _drafts(parent=None)}):
        assert call(**kw) == INVALID, kw
    assert call(nb=255) == CAPACITY
    assert call(d=_drafts(n_trees=0), row0=None, ids=None, first=None) == cdb.CDB_OK


def test_tree_commit_refusals():
    full = cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 1, 1)

    def call(desc=DESC, kv=full, d=_drafts(), out=tree.cdb_accepted(1, 1, None), ws=1, nb=BIG):
        return _status("cdb_tree_commit", desc, kv, d, out, ws, nb, None)

    for kw in ({"kv": None}, {"out": None}, {"ws": None}, {"d": _drafts(seq=None)}, {"d": _drafts(len=None)},
               {"out": tree.cdb_accepted(None, 1, 1)}, {"out": tree.cdb_accepted(1, None, 1)},
               {"kv": cdb.cdb_kv(1, None, 1, 1, 1, 1, 1, 1, 1)}, {"kv": cdb.cdb_kv(1, 1, 1, 1, 1, -1, 1, 1, 1)},
               {"kv": cdb.cdb_kv(1, 1, 1, 1, 1, 1, None, 1, 1)}, {"kv": cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, -1, 1)}):
        assert call(**kw) == INVALID, kw
    assert call(desc=BAD_DESC) == UNSUPPORTED
    assert call(kv=cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 1, 1 << 28)) == CAPACITY
    assert call(nb=255) == CAPACITY
    assert call(d=_drafts(n_trees=0)) == cdb.CDB_OK


def test_tree_attention_refusals():
    full = cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 4, 8)
    see = tree.cdb_tree(8, 1, 1, None)
    need = tree.cdb_tree_workspace_bytes(DESC, 8, 0)

    def call(desc=DESC, kv=full, rows=cdb.cdb_rows(8, 1, 1, 1, 1), t=see, stage=1, layer=0, q=1, out=1, ws=1, nb=need):
        return _status("cdb_tree_attention", desc, kv, rows, t, stage, layer, q, out, ws, nb, None)

    for kw in ({"desc": None}, {"kv": None}, {"rows": None}, {"t": None}, {"q": None}, {"out": None}, {"ws": None},
               {"t": tree.cdb_tree(0, 1, 1, 1)}, {"t": tree.cdb_tree(65, 1, 1, 1)}, {"t": tree.cdb_tree(8, None, 1, 1)},
               {"t": tree.cdb_tree(8, 1, None, 1)}, {"stage": 3}, {"stage": -1}, {"layer": 2}, {"layer": -1},
               {"rows": cdb.cdb_rows(-1, 1, 1, 1, 1)}, {"rows": cdb.cdb_rows(8, 1, None, 1, 1)},
               {"rows": cdb.cdb_rows(8, 1, 1, 1, None)}, {"kv": cdb.cdb_kv(1, None, 1, 1, 1, 1, 1, 4, 8)},
               {"kv": cdb.cdb_kv(1, 1, 1, 1, 1, 1, None, 4, 8)}, {"kv": cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, -4, 8)},
               {"kv": cdb.cdb_kv(1, 1, 1, 1, 0, 1, 1, 4, 8)}):
        assert call(**kw) == INVALID, kw
    assert call(desc=BAD_DESC) == UNSUPPORTED
    assert call(rows=cdb.cdb_rows(cdb.MAX_ROWS + 1, 1, 1, 1, 1)) == CAPACITY
    assert call(kv=cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 4, 1 << 28)) == CAPACITY
    assert call(nb=255) == CAPACITY
    assert call(rows=cdb.cdb_rows(0, 1, 1, 1, 1)) == cdb.CDB_OK


def test_tree_stage_refusals():
    """On top of what the plain stage calls refuse."""
    model, state = cdb.cdb_model(1, DESC), cdb.cdb_state(1, None, 4)
    kv = cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 4, 8)
    rows, out, good = cdb.cdb_rows(8, 1, 1, 1, 1, 1), cdb.cdb_step_out(1, 1, 1, 1, 1), tree.cdb_tree(8, 1, 1, 1)
    nb = tree.cdb_tree_workspace_bytes(DESC, 8, 0)

    def calls(t, nb=nb, kv=kv):
        return [_status("cdb_tree_prelude", model, kv, state, rows, t, 1, 1, nb, None),
                _status("cdb_tree_step", model, kv, state, rows, t, None, out, 1, nb, None),
                _status("cdb_tree_coda", model, kv, state, rows, t, 1, 1, 1, nb, None)]

    for t in (None, tree.cdb_tree(0, 1, 1, 1), tree.cdb_tree(65, 1, 1, 1), tree.cdb_tree(8, None, 1, 1),
              tree.cdb_tree(8, 1, None, 1), tree.cdb_tree(8, 1, 1, None)):
        assert calls(t) == [INVALID] * 3
    assert calls(good, nb=cdb.cdb_workspace_bytes(DESC, 1)) == [CAPACITY] * 3
    assert calls(good, kv=cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 4, 1 << 28)) == [CAPACITY] * 3
    assert calls(good, kv=cdb.cdb_kv(1, 1, 1, 0, 0, 0, 1, 4, 8)) == [INVALID] * 3
    bad = cdb.cdb_gate(0.5, 1, None)
    assert _status("cdb_tree_step", model, kv, state, rows, good, bad, out, 1, nb, None) == INVALID


def test_holders_refuse_tensors_on_the_host():
    i = torch.zeros(4, dtype=torch.int32)
    m = torch.zeros(4, dtype=torch.int64)
    for make in (lambda: tree.Tree(4, i, m, i), lambda: tree.PagePool(i, i[:1]),
                 lambda: tree.Drafts(i, i, i, i.view(4, 1), i.view(4, 1))):
        with pytest.raises(cdb.CdbError) as e:
            make()
        assert e.value.status == INVALID


def test_calls_stay_on_the_current_device(monkeypatch):
    """A workspace or a stream of another device is refused before anything is enqueued."""
    class On:
        def __init__(self, index, cuda_stream=7):
            self.device, self.cuda_stream = torch.device("cuda", index), cuda_stream

        def data_ptr(self):
            return 1

        def numel(self):
            return BIG

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert tree._stream("f", On(0), On(0)) == 7
    d, out, acc = _drafts(n_trees=0), tree.cdb_row_map(8, *[1] * 8), tree.cdb_accepted(1, 1, 1)
    for ws, stream in ((On(1), None), (On(0), On(1)), (On(1), On(1))):
        for call in (lambda: tree.cdb_tree_rows(d, out, ws, stream),
                     lambda: tree.cdb_tree_commit(DESC, cdb.cdb_kv(1, 1, 1, 1, 1, 1, 1, 1, 1), d, acc, ws, stream)):
            with pytest.raises(cdb.CdbError) as e:
                call()
            assert e.value.status == INVALID
