"""Python binding of libcdb's verification of drafted tokens (include/libcdb_tree.h): page tables from sequence lengths,
drafted trees as rows, their attention and stage calls, greedy acceptance, and the move of the accepted K/V.

Argument marshalling only; the calls run in the HIP kernels of libcdb.so.  The holder classes check their tensors (device,
type, size, contiguity) and raise CdbError(CDB_ERR_INVALID_ARG); the calls take their C structs, as those of the package do
(each struct keeps its tensors alive).
"""
from __future__ import annotations

import ctypes as C

import torch

from . import (CDB_ERR_CAPACITY, CDB_ERR_INVALID_ARG, MAX_ROWS, CdbError, _check, _ptr, cdb_kv, cdb_model,
               cdb_model_desc, cdb_rows, cdb_state, cdb_step_out, cdb_workspace_init, lib as _lib)

EXPORTED = ("cdb_tree_workspace_bytes", "cdb_map_pages", "cdb_tree_rows", "cdb_tree_attention", "cdb_tree_prelude",
            "cdb_tree_step", "cdb_tree_coda", "cdb_tree_accept", "cdb_tree_commit")

MAX_NODES, MAX_TREES = 64, 256
KV_FULL, KV_SHARED, KV_FIRST_THEN_SHARED = 0, 1, 2
CDB_DEV_NO_PAGES = 4


class cdb_tree(C.Structure):
    _fields_ = [("max_nodes", C.c_int32), ("base", C.c_void_p), ("mask", C.c_void_p), ("rope_pos", C.c_void_p)]


class cdb_page_pool(C.Structure):
    _fields_ = [("free_ids", C.c_void_p), ("free_count", C.c_void_p), ("capacity", C.c_int32)]


class cdb_drafts(C.Structure):
    _fields_ = [("n_trees", C.c_int32), ("max_nodes", C.c_int32), ("max_seqs", C.c_int32), ("seq", C.c_void_p),
                ("len", C.c_void_p), ("n_nodes", C.c_void_p), ("parent", C.c_void_p), ("tokens", C.c_void_p)]


class cdb_row_map(C.Structure):
    _fields_ = [("capacity", C.c_int32), ("row0", C.c_void_p), ("n_rows", C.c_void_p), ("seq", C.c_void_p),
                ("pos", C.c_void_p), ("base", C.c_void_p), ("rope_pos", C.c_void_p), ("tokens", C.c_void_p),
                ("mask", C.c_void_p)]


class cdb_accepted(C.Structure):
    _fields_ = [("path", C.c_void_p), ("count", C.c_void_p), ("next", C.c_void_p)]


_bound = False


def lib() -> C.CDLL:
    global _bound
    L = _lib()
    if not _bound:
        P, I, S = C.c_void_p, C.c_int32, C.c_size_t
        L.cdb_tree_workspace_bytes.argtypes = [P, I, I]
        L.cdb_tree_workspace_bytes.restype = S
        L.cdb_map_pages.argtypes = [P, P, I, I, P, P, P, I, P, P, P, S, P]
        L.cdb_tree_rows.argtypes = [P, P, P, S, P]
        L.cdb_tree_attention.argtypes = [P, P, P, P, I, I, P, P, P, S, P]
        L.cdb_tree_prelude.argtypes = [P, P, P, P, P, P, P, S, P]
        L.cdb_tree_step.argtypes = [P, P, P, P, P, P, P, P, S, P]
        L.cdb_tree_coda.argtypes = [P, P, P, P, P, P, P, P, S, P]
        L.cdb_tree_accept.argtypes = [P, P, P, I, P, P, P, S, P]
        L.cdb_tree_commit.argtypes = [P, P, P, P, P, S, P]
        for f in EXPORTED[1:]:
            getattr(L, f).restype = C.c_int
        _bound = True
    return L


def _stream(fn, stream, ws) -> int:
    """The stream's handle.  Workspace and stream belong to the current device, on which the kernels run.  The current
    stream is looked up without making a Stream object, which would take longer than the smaller of these calls run."""
    here = torch.cuda.current_device()
    if ws.device.index != here or (stream is not None and stream.device.index != here):
        raise CdbError(fn, CDB_ERR_INVALID_ARG)
    return torch._C._cuda_getCurrentRawStream(here) if stream is None else stream.cuda_stream


def _need(fn, ok):
    if not ok:
        raise CdbError(fn, CDB_ERR_INVALID_ARG)


def _tensor(fn, t, dtype, *shape):
    """A contiguous device tensor of this type; shape: its sizes (None: any)."""
    _need(fn, isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.is_contiguous() and
          (not shape or (t.dim() == len(shape) and all(w is None or n == w for n, w in zip(t.shape, shape)))))
    return t


def _flat(fn, t, dtype, least):
    """The address of a contiguous device tensor of this type with at least so many values."""
    if not (t.is_cuda and t.dtype is dtype and t.numel() >= least and t.is_contiguous()):
        raise CdbError(fn, CDB_ERR_INVALID_ARG)
    return t.data_ptr()


# ---------------------------------------------------------------- C ABI, same names

def cdb_tree_workspace_bytes(desc: cdb_model_desc, max_rows: int, max_seqs: int) -> int:
    return lib().cdb_tree_workspace_bytes(C.byref(desc), max_rows, max_seqs)


def _ref(c):
    return None if c is None else C.byref(c)


def cdb_map_pages(desc: cdb_model_desc, page_table, pre, core, coda, kv_layout: int, length, mapped, ws, stream=None):
    """page_table: device int32 [max_seqs][r_max + 2][max_pages]; pre, core, coda: cdb_page_pool, None for a stage
    without layers; length, mapped: device int32 [max_seqs]."""
    _tensor("cdb_map_pages", page_table, torch.int32, None, desc.r_max + 2, None)
    S, _, P = page_table.shape
    lens, have = (_flat("cdb_map_pages", t, torch.int32, S) for t in (length, mapped))
    _check("cdb_map_pages", lib().cdb_map_pages(C.byref(desc), page_table.data_ptr(), S, P, _ref(pre), _ref(core),
                                                _ref(coda), kv_layout, lens, have, ws.data_ptr(), ws.numel(),
                                                _stream("cdb_map_pages", stream, ws)))


def _trees_fit(fn, drafts, holder):
    """Whether the buffers of a holder's struct are for these trees (structs made by hand are taken as they are)."""
    _need(fn, getattr(holder, "trees", drafts.n_trees) >= drafts.n_trees)
    _need(fn, getattr(holder, "nodes", drafts.max_nodes) == drafts.max_nodes)


def _rows_fit(fn, rows, tree):
    _need(fn, getattr(tree, "n_rows", rows.n_rows) >= rows.n_rows)


def cdb_tree_rows(drafts: cdb_drafts, out: cdb_row_map, ws, stream=None):
    _trees_fit("cdb_tree_rows", drafts, out)
    _check("cdb_tree_rows", lib().cdb_tree_rows(C.byref(drafts), C.byref(out), _ptr(ws), ws.numel(), _stream("cdb_tree_rows", stream, ws)))


def cdb_tree_attention(desc: cdb_model_desc, kv: cdb_kv, rows: cdb_rows, tree: cdb_tree, stage: int, layer: int, q, out,
                       ws, stream=None):
    """q: device fp32 [n_rows][d]; out: device bf16 in fragment order (cdb_paged_attention)."""
    n = rows.n_rows
    padded = 32 if n <= 32 else 64 if n <= 64 else 128 if n <= 128 else max(n, 256)
    _rows_fit("cdb_tree_attention", rows, tree)
    qp = _flat("cdb_tree_attention", q, torch.float32, n * desc.d)
    op = _flat("cdb_tree_attention", out, torch.bfloat16, padded * desc.d)
    _check("cdb_tree_attention", lib().cdb_tree_attention(C.byref(desc), C.byref(kv), C.byref(rows), C.byref(tree), stage,
                                                          layer, qp, op, ws.data_ptr(), ws.numel(), _stream("cdb_tree_attention", stream, ws)))


def cdb_tree_prelude(model: cdb_model, kv: cdb_kv, state: cdb_state, rows: cdb_rows, tree: cdb_tree, tokens, ws,
                     stream=None):
    _rows_fit("cdb_tree_prelude", rows, tree)
    _check("cdb_tree_prelude", lib().cdb_tree_prelude(C.byref(model), C.byref(kv), C.byref(state), C.byref(rows),
                                                      C.byref(tree), _ptr(tokens), _ptr(ws), ws.numel(),
                                                      _stream("cdb_tree_prelude", stream, ws)))


def cdb_tree_step(model: cdb_model, kv: cdb_kv, state: cdb_state, rows: cdb_rows, tree: cdb_tree, out: cdb_step_out, ws,
                  stream=None, gate=None):
    """gate: cdb_gate for exits by a threshold, None for replayed depths."""
    _rows_fit("cdb_tree_step", rows, tree)
    _check("cdb_tree_step", lib().cdb_tree_step(C.byref(model), C.byref(kv), C.byref(state), C.byref(rows),
                                                C.byref(tree), _ref(gate), C.byref(out), _ptr(ws), ws.numel(),
                                                _stream("cdb_tree_step", stream, ws)))


def cdb_tree_coda(model: cdb_model, kv: cdb_kv, state: cdb_state, rows: cdb_rows, tree: cdb_tree, logits, next_ids, ws,
                  stream=None):
    _rows_fit("cdb_tree_coda", rows, tree)
    _check("cdb_tree_coda", lib().cdb_tree_coda(C.byref(model), C.byref(kv), C.byref(state), C.byref(rows),
                                                C.byref(tree), _ptr(logits), _ptr(next_ids), _ptr(ws), ws.numel(),
                                                _stream("cdb_tree_coda", stream, ws)))


def cdb_tree_accept(drafts: cdb_drafts, row0, next_ids, first_ids, out: cdb_accepted, ws, stream=None):
    """row0, first_ids: device int32 [n_trees]; next_ids: device int32, by row.  drafts: seq and length as cdb_tree_rows got
    them, so that trees it refused are known."""
    _trees_fit("cdb_tree_accept", drafts, out)
    T = drafts.n_trees
    at, first = (_flat("cdb_tree_accept", t, torch.int32, T) for t in (row0, first_ids))
    ids = _flat("cdb_tree_accept", next_ids, torch.int32, 0)
    _check("cdb_tree_accept", lib().cdb_tree_accept(C.byref(drafts), at, ids, next_ids.numel(), first, C.byref(out),
                                                    ws.data_ptr(), ws.numel(), _stream("cdb_tree_accept", stream, ws)))


def cdb_tree_commit(desc: cdb_model_desc, kv: cdb_kv, drafts: cdb_drafts, accepted: cdb_accepted, ws, stream=None):
    _trees_fit("cdb_tree_commit", drafts, accepted)
    _check("cdb_tree_commit", lib().cdb_tree_commit(C.byref(desc), C.byref(kv), C.byref(drafts), C.byref(accepted),
                                                    _ptr(ws), ws.numel(), _stream("cdb_tree_commit", stream, ws)))


# ---------------------------------------------------------------- device-memory holders (torch)

def _held(c, *tensors, **sizes):
    """The struct with its tensors, which live as long as it does, and their sizes, which the calls check."""
    c.keep = tensors
    for k, v in sizes.items():
        setattr(c, k, v)
    return c


class TreeWorkspace:
    """Scratch of the calls above, and of the package's stage calls, for up to max_rows rows and max_seqs sequences."""

    def __init__(self, desc: cdb_model_desc, max_rows: int, max_seqs: int, device="cuda", stream=None):
        n = cdb_tree_workspace_bytes(desc, max_rows, max_seqs)
        if n == 0:
            raise CdbError("cdb_tree_workspace_bytes", CDB_ERR_CAPACITY)
        self.buf = torch.empty(n, dtype=torch.uint8, device=device)
        cdb_workspace_init(self.buf, stream)


class Tree:
    """What drafted rows see (cdb_tree): base and rope_pos int32, mask int64 (64 bits), one entry per row.  For rows
    laid out by cdb_tree_rows: TreeRows.tree()."""

    def __init__(self, max_nodes: int, base, mask, rope_pos):
        n = base.numel()
        self.base, self.rope_pos = _tensor("Tree", base, torch.int32, n), _tensor("Tree", rope_pos, torch.int32, n)
        self.mask = _tensor("Tree", mask, torch.int64, n)
        self.c = _held(cdb_tree(max_nodes, _ptr(base), _ptr(mask), _ptr(rope_pos)), base, mask, rope_pos, n_rows=n)


class PagePool:
    """A pool's free pages (cdb_page_pool): free_ids int32 [capacity], the next page at free_ids[count - 1]; free_count
    int32 [1].  PagePool.full(n): all n pages free, page 0 next."""

    def __init__(self, free_ids, free_count):
        self.free_ids, self.free_count = _tensor("PagePool", free_ids, torch.int32, None), \
            _tensor("PagePool", free_count, torch.int32, 1)
        self.c = _held(cdb_page_pool(_ptr(free_ids), _ptr(free_count), free_ids.numel()), free_ids, free_count)

    @classmethod
    def full(cls, n: int, device="cuda"):
        return cls(torch.arange(n - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.tensor([n], dtype=torch.int32, device=device))


class Drafts:
    """Drafted trees (cdb_drafts), int32: seq, n_nodes [n_trees]; length [max_seqs], by sequence; parent, tokens
    [n_trees][max_nodes]."""

    def __init__(self, seq, length, n_nodes, parent, tokens):
        _need("Drafts", seq.dim() == 1 and parent.dim() == 2)
        (T, N), S = parent.shape, length.numel()
        self.seq, self.n_nodes = _tensor("Drafts", seq, torch.int32, T), _tensor("Drafts", n_nodes, torch.int32, T)
        self.length = _tensor("Drafts", length, torch.int32, S)
        self.parent, self.tokens = _tensor("Drafts", parent, torch.int32, T, N), _tensor("Drafts", tokens, torch.int32, T, N)
        arrays = (seq, length, n_nodes, parent, tokens)
        self.c = _held(cdb_drafts(T, N, S, *(_ptr(t) for t in arrays)), *arrays)


class TreeRows:
    """Buffers that cdb_tree_rows fills (cdb_row_map).  rows(slot, ...) and tree(max_nodes) give the arguments of a stage
    call over them, at capacity with the row count in device memory."""

    def __init__(self, n_trees: int, capacity: int, device="cuda"):

        def ints(n, dtype=torch.int32):
            return torch.zeros(n, dtype=dtype, device=device)

        self.capacity = capacity
        self.row0, self.n_rows = ints(n_trees), ints(1)
        self.seq, self.pos, self.base, self.rope_pos, self.tokens = (ints(capacity) for _ in range(5))
        self.mask = ints(capacity, torch.int64)
        arrays = (self.row0, self.n_rows, self.seq, self.pos, self.base, self.rope_pos, self.tokens, self.mask)
        self.c = _held(cdb_row_map(capacity, *(_ptr(t) for t in arrays)), *arrays, trees=n_trees)

    def rows(self, slot, c=None, depth=None):
        from . import Rows
        return Rows(slot, self.seq, self.pos, c, depth, device=self.seq.device, d_n_rows=self.n_rows)

    def tree(self, max_nodes: int) -> Tree:
        return Tree(max_nodes, self.base, self.mask, self.rope_pos)


class Accepted:
    """Accepted paths (cdb_accepted): path [n_trees][max_nodes], count and next [n_trees]."""

    def __init__(self, n_trees: int, max_nodes: int, device="cuda"):
        self.path = torch.full((n_trees, max_nodes), -1, dtype=torch.int32, device=device)
        self.count = torch.zeros(n_trees, dtype=torch.int32, device=device)
        self.next = torch.zeros(n_trees, dtype=torch.int32, device=device)
        arrays = (self.path, self.count, self.next)
        self.c = _held(cdb_accepted(*(_ptr(t) for t in arrays)), *arrays, trees=n_trees, nodes=max_nodes)
