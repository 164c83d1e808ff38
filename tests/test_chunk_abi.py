"""The C entries of include/libcdb_chunk.h and the sampled acceptance of include/libcdb_tree.h: exported, and bad arguments
refused before anything is enqueued; the Python holders refuse tensors that the kernels could not read.  CPU only (no call
here reaches a launch)."""
import ctypes as C
import os
import re

import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk, tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DESC = cdb.make_desc(cdbgen.TINY)
BAD_DESC = cdb.make_desc(cdbgen.shrink(cdbgen.TINY, head_dim=80, n_heads=4, d=320))
BIG = 1 << 40
INVALID, CAPACITY, UNSUPPORTED = cdb.CDB_ERR_INVALID_ARG, cdb.CDB_ERR_CAPACITY, cdb.CDB_ERR_UNSUPPORTED
KV = cdb.cdb_kv(16, 16, 16, 1, 1, 1, 16, 4, 8)


def _status(fn, *args):
    L = chunk.lib() if fn in chunk.EXPORTED else tree.lib()
    return getattr(L, fn)(*(C.byref(a) if isinstance(a, C.Structure) else a for a in args))


def test_every_declared_entry_is_exported():
    text = open(os.path.join(ROOT, "include", "libcdb_chunk.h")).read()
    names = re.findall(r"^(?:cdb_status|size_t)\s+(cdb_\w+)\s*\(", text, re.M)
    assert sorted(names) == sorted(chunk.EXPORTED)
    for n in names:
        assert hasattr(chunk.lib(), n), n


@pytest.mark.parametrize("shape", [cdbgen.TINY, cdbgen.OURO, cdbgen.HUGINN], ids=lambda s: s.name)
def test_workspace_serves_every_smaller_call(shape):
    desc = cdb.make_desc(shape)
    sizes = [chunk.cdb_chunk_workspace_bytes(desc, r, 8) for r in (*range(600), 4095, 4096, 4097, 65535, 65536)]
    assert all(b >= a for a, b in zip(sizes, sizes[1:])) and sizes[0] >= 256
    for rows, chunks in ((65537, 1), (-1, 1), (1, 257), (1, -1)):
        assert chunk.cdb_chunk_workspace_bytes(desc, rows, chunks) == 0
    assert chunk.cdb_chunk_workspace_bytes(BAD_DESC, 1, 1) == 0
    # a tree workspace holds what sampled acceptance needs
    for rows in (0, 1, 256):
        nb = tree.cdb_tree_workspace_bytes(desc, rows, 1)
        assert _sample(desc=desc, n_trees=0, n_rows=rows, ls=shape.vocab, ds=shape.vocab, nb=nb) == cdb.CDB_OK



def _chunks(**kw):
    a = dict(n_chunks=2, n_rows=8, row0=16, seq=16, pos0=16, c=16)
    a.update(kw)
    return chunk.cdb_chunks(*a.values())


def _qkv(**kw):
    a = dict(q=1 << 20, k=2 << 20, v=3 << 20, type=1, norm=1, q_stride=256, k_stride=256, v_stride=256, q_gain=None, k_gain=None, rope=None)
    a.update(kw)
    return chunk.cdb_qkv(*a.values())


def _write(desc=DESC, kv=KV, ch=_chunks(), stage=1, layer=0, qkv=_qkv(), q=16, q_type=1, ws=16, nb=256):
    return _status("cdb_chunk_qkv", desc, kv, ch, stage, layer, qkv, q, q_type, ws, nb, None)


def _attend(desc=DESC, kv=KV, ch=_chunks(), stage=1, layer=0, q=16, q_type=1, out=1 << 20, order=1, ws=16, nb=BIG):
    return _status("cdb_chunk_attention", desc, kv, ch, stage, layer, q, q_type, out, order, ws, nb, None)


@pytest.mark.parametrize("call", [_write, _attend], ids=["qkv", "attention"])
def test_bad_chunks_are_refused_alike(call):
    for kw in ({"desc": None}, {"kv": None}, {"ch": None}, {"ws": None}, {"stage": 3}, {"stage": -1}, {"layer": 2},
               {"layer": -1}, {"q_type": 2}, {"q_type": -1}, {"ch": _chunks(n_chunks=-1)}, {"ch": _chunks(n_rows=-1)},
               {"ch": _chunks(row0=None)}, {"ch": _chunks(seq=None)}, {"ch": _chunks(pos0=None)}, {"ch": _chunks(c=None)},
               {"kv": cdb.cdb_kv(16, None, 16, 1, 1, 1, 16, 4, 8)}, {"kv": cdb.cdb_kv(16, 16, 16, 1, 0, 1, 16, 4, 8)},
               {"kv": cdb.cdb_kv(16, 16, 16, 1, 1, 1, None, 4, 8)}, {"kv": cdb.cdb_kv(16, 16, 16, 1, 1, 1, 16, -4, 8)},
               {"kv": cdb.cdb_kv(16, 16, 16, 1, 1, 1, 16, 4, -8)}, {"q": None}, {"q": 8}):
        assert call(**kw) == INVALID, kw
    assert call(desc=BAD_DESC) == UNSUPPORTED
    for kw in ({"ch": _chunks(n_chunks=257)}, {"ch": _chunks(n_rows=65537)}, {"nb": 255},
               {"kv": cdb.cdb_kv(16, 16, 16, 1, 1, 1, 16, 4, 1 << 28)}):
        assert call(**kw) == CAPACITY, kw
    assert call(ch=_chunks(n_rows=0)) == cdb.CDB_OK
    assert call(ch=_chunks(n_chunks=0, seq=None, pos0=None, c=None)) == cdb.CDB_OK


def test_qkv_refusals():
    for kw in ({"q": None}, {"k": None}, {"v": None}, {"type": 2}, {"type": -1}, {"norm": 2}, {"q_stride": 255},
               {"k_stride": 260}, {"v_stride": 0}, {"v_stride": -256}, {"q": 8}, {"k": 24}, {"v": 4}, {"q_gain": 8},
               {"k_gain": 2}):
        assert _write(qkv=_qkv(**kw)) == INVALID, kw
    assert _write(qkv=_qkv(type=0, q_stride=258)) == INVALID
    assert _write(qkv=None) == INVALID
    # q_out in part of what is read: 8 rows of 256 bf16 values are 4096 bytes
    for q, kw in ((2 << 20, {}), ((2 << 20) + 4080, {}), ((3 << 20) - 4080, {}), ((1 << 20) + 16, {}), (1 << 20, {"q_stride": 768}),
                  (1 << 20, {"type": 0}), ((3 << 20) + 7 * 1536 + 496, {"v_stride": 768}), (4096, {"q": 4096 + 4080})):
        assert _write(q=q, qkv=_qkv(**kw)) == INVALID, (q, kw)
    assert _write(q=1 << 20, q_type=0) == INVALID


def test_attention_refusals():
    need = chunk.cdb_chunk_workspace_bytes(DESC, 8, 2)
    for kw in ({"out": None}, {"out": 24}, {"order": 2}, {"order": -1}):
        assert _attend(**kw) == INVALID, kw
    assert _attend(nb=need - 1) == CAPACITY
    for kw in ({"out": 16}, {"out": 4096}, {"out": 8192, "q_type": 0}, {"out": 1 << 20, "q": (1 << 20) + 16384 - 16, "order": 0}):
        assert _attend(**kw) == INVALID, kw


def _sample(desc=DESC, n_trees=2, n_rows=8, row0=16, first=16, out=tree.cdb_accepted(16, 16, 16), ws=16, nb=BIG, sm=True,
            d=None, **kw):
    s = dict(logits=16, draft=16, ls=1024, ds=1024, t=None, dt=None, u=16, un=16)
    s.update(kw)
    d = d or tree.cdb_drafts(n_trees, 8, 4, None, None, 16, 16, 16)
    return _status("cdb_tree_sample", desc, d, row0, n_rows, first, tree.cdb_sampling(*s.values()) if sm else None, out, ws,
                   nb, None)


def test_tree_sample_refusals():
    for kw in ({"desc": None}, {"row0": None}, {"first": None}, {"out": None}, {"ws": None}, {"n_rows": -1}, {"sm": None},
               {"out": tree.cdb_accepted(None, 16, 16)}, {"out": tree.cdb_accepted(16, None, 16)},
               {"out": tree.cdb_accepted(16, 16, None)}, {"logits": None}, {"logits": 8}, {"draft": 8}, {"ls": 1020},
               {"ls": 1026}, {"ds": 1020}, {"ds": 1026}, {"u": None}, {"un": None}, {"n_trees": -1},
               {"d": tree.cdb_drafts(2, 8, 4, None, None, 16, None, 16)}, {"d": tree.cdb_drafts(2, 65, 4, None, None, 16, 16, 16)}):
        assert _sample(**kw) == INVALID, kw
    assert _sample(desc=BAD_DESC) == UNSUPPORTED
    assert _sample(desc=cdb.make_desc(cdbgen.shrink(cdbgen.TINY, vocab=(1 << 20) + 32))) == UNSUPPORTED
    for kw in ({"n_rows": 257}, {"nb": 255}, {"n_trees": 257}):
        assert _sample(**kw) == CAPACITY, kw
    assert _sample(n_trees=0, row0=None, first=None) == cdb.CDB_OK


def test_holders_refuse_tensors_on_the_host():
    i, x, b = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64), torch.zeros(64, dtype=torch.bfloat16)
    f = torch.zeros(4, 32)
    for make in (lambda: chunk.Chunks(4, i, i[:3], i[:3]), lambda: chunk.QKV(x, x, x), lambda: chunk.QKV(x[0], x[0], x[0]),
                 lambda: chunk.QKV(x, x, x, q_gain=b), lambda: tree.Sampling(f, f, f[0])):
        with pytest.raises(cdb.CdbError) as e:
            make()
        assert e.value.status == INVALID
