"""Python binding of libcdb's calls over chunks of new tokens (include/libcdb_chunk.h): queries, keys and values normalised,
rotated and written to the paged cache, and causal attention over it.

Argument marshalling only; the calls run in the HIP kernels of libcdb.so.  The holder classes check their tensors (device,
type, size, strides) and raise CdbError(CDB_ERR_INVALID_ARG); the calls take their C structs, which keep the tensors alive.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import CDB_ERR_CAPACITY, CDB_ERR_INVALID_ARG, CdbError, _check, _ptr, cdb_kv, cdb_model_desc, cdb_workspace_init, lib as _lib
from .tree import _held, _here, _need, _stream, _tensor

EXPORTED = ("cdb_chunk_workspace_bytes", "cdb_chunk_qkv", "cdb_chunk_attention")

MAX_CHUNKS, MAX_CHUNK_ROWS = 256, 65536
CDB_F32, CDB_BF16 = 0, 1
CDB_ORDER_FRAGMENTS, CDB_ORDER_ROWS = 0, 1
_TYPES = {torch.float32: CDB_F32, torch.bfloat16: CDB_BF16}


class cdb_chunks(C.Structure):
    _fields_ = [("n_chunks", C.c_int32), ("n_rows", C.c_int32), ("row0", C.c_void_p), ("seq", C.c_void_p),
                ("pos0", C.c_void_p), ("c", C.c_void_p)]


class cdb_qkv(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("type", C.c_int32), ("norm", C.c_int32),
                ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("v_stride", C.c_int64), ("q_gain", C.c_void_p),
                ("k_gain", C.c_void_p), ("rope_pos", C.c_void_p)]


_bound = False


def lib() -> C.CDLL:
    global _bound
    L = _lib()
    if not _bound:
        P, I, S = C.c_void_p, C.c_int32, C.c_size_t
        L.cdb_chunk_workspace_bytes.argtypes = [P, I, I]
        L.cdb_chunk_workspace_bytes.restype = S
        L.cdb_chunk_qkv.argtypes = [P, P, P, I, I, P, P, I, P, S, P]
        L.cdb_chunk_attention.argtypes = [P, P, P, I, I, P, I, P, I, P, S, P]
        for f in EXPORTED[1:]:
            getattr(L, f).restype = C.c_int
        _bound = True
    return L


# ---------------------------------------------------------------- C ABI, same names

def cdb_chunk_workspace_bytes(desc: cdb_model_desc, max_rows: int, max_chunks: int) -> int:
    return lib().cdb_chunk_workspace_bytes(C.byref(desc), max_rows, max_chunks)


def _rows(fn, t, dtype, least, here) -> int:
    """The address of a contiguous tensor of device `here`, of this type (None: fp32 or bf16) with at least so many values."""
    if not ((t.dtype is dtype if dtype else t.dtype in _TYPES) and t.is_cuda and t.get_device() == here and
            t.numel() >= least and t.is_contiguous()):
        raise CdbError(fn, CDB_ERR_INVALID_ARG)
    return t.data_ptr()


def cdb_chunk_qkv(desc: cdb_model_desc, kv: cdb_kv, chunks: cdb_chunks, stage: int, layer: int, qkv: cdb_qkv, q_out, ws,
                  stream=None):
    """q_out: device fp32 or bf16 [n_rows][d]."""
    fn, n, d = "cdb_chunk_qkv", chunks.n_rows, desc.d
    shape = getattr(qkv, "shape", None)  # structs made by hand are taken as they are
    if shape is not None and (shape[0] < n or shape[1] != desc.n_heads or shape[2] != desc.head_dim):
        raise CdbError(fn, CDB_ERR_INVALID_ARG)
    to = _rows(fn, q_out, None, n * d, _here(fn, ws, chunks, qkv))
    _check(fn, lib().cdb_chunk_qkv(C.byref(desc), C.byref(kv), C.byref(chunks), stage, layer, C.byref(qkv), to,
                                   _TYPES[q_out.dtype], ws.data_ptr(), ws.numel(), _stream(fn, stream, ws)))


def cdb_chunk_attention(desc: cdb_model_desc, kv: cdb_kv, chunks: cdb_chunks, stage: int, layer: int, q, out, ws,
                        stream=None, order: int = CDB_ORDER_ROWS):
    """q: device fp32 or bf16 [n_rows][d]; out: device bf16 [n_rows][d], or, in CDB_ORDER_FRAGMENTS, of n_rows rounded up to
    32 rows."""
    fn, n, d = "cdb_chunk_attention", chunks.n_rows, desc.d
    here = _here(fn, ws, chunks)
    at = _rows(fn, q, None, n * d, here)
    to = _rows(fn, out, torch.bfloat16, (n if order == CDB_ORDER_ROWS else (n + 31) // 32 * 32) * d, here)
    _check(fn, lib().cdb_chunk_attention(C.byref(desc), C.byref(kv), C.byref(chunks), stage, layer, at, _TYPES[q.dtype], to,
                                         order, ws.data_ptr(), ws.numel(), _stream(fn, stream, ws)))


# ---------------------------------------------------------------- device-memory holders (torch)

class ChunkWorkspace:
    """Scratch of the calls above for up to max_rows rows in max_chunks chunks."""

    def __init__(self, desc: cdb_model_desc, max_rows: int, max_chunks: int, device="cuda", stream=None):
        n = cdb_chunk_workspace_bytes(desc, max_rows, max_chunks)
        if n == 0:
            raise CdbError("cdb_chunk_workspace_bytes", CDB_ERR_CAPACITY)
        self.buf = torch.empty(n, dtype=torch.uint8, device=device)
        cdb_workspace_init(self.buf, stream)


class Chunks:
    """The chunks of a call (cdb_chunks), int32: row0 [n_chunks + 1], seq, pos0 and, for the core, c [n_chunks].  n_rows: what
    the row buffers hold."""

    def __init__(self, n_rows: int, row0, seq, pos0, c=None):
        n = seq.numel()
        _need("Chunks", n_rows >= 0)
        self.row0 = _tensor("Chunks", row0, torch.int32, n + 1)
        self.seq, self.pos0 = (_tensor("Chunks", t, torch.int32, n) for t in (seq, pos0))
        self.cc = None if c is None else _tensor("Chunks", c, torch.int32, n)
        self.c = _held(cdb_chunks(n, n_rows, _ptr(row0), _ptr(seq), _ptr(pos0), _ptr(c)), row0, seq, pos0, c)


class QKV:
    """Queries, keys and values of a call's rows (cdb_qkv): fp32 or bf16 [n_rows][heads][head_dim], each row contiguous,
    rows any multiple of 16 bytes apart (parts of a fused projection: qkv.unbind(1)).  norm: RMSNorm of every query and key
    head, with gains bf16 [head_dim] (None: 1).  rope_pos: int32 [n_rows], None: the rows' own positions."""

    def __init__(self, q, k, v, norm: bool = False, q_gain=None, k_gain=None, rope_pos=None):
        _need("QKV", q.dim() == 3 and q.dtype in _TYPES)
        n, H, hd = q.shape
        for t in (q, k, v):
            _need("QKV", t.is_cuda and t.dtype is q.dtype and t.shape == q.shape and
                  (t.numel() == 0 or (t.stride(2) == 1 and (H == 1 or t.stride(1) == hd))))
        for t in (q_gain, k_gain):
            _need("QKV", t is None or _tensor("QKV", t, torch.bfloat16, hd) is t)
        _need("QKV", rope_pos is None or _tensor("QKV", rope_pos, torch.int32, n) is rope_pos)
        strides = [t.stride(0) if n > 1 else H * hd for t in (q, k, v)]  # of one row any
        self.q, self.k, self.v, self.q_gain, self.k_gain, self.rope_pos = q, k, v, q_gain, k_gain, rope_pos
        self.c = _held(cdb_qkv(_ptr(q), _ptr(k), _ptr(v), _TYPES[q.dtype], int(bool(norm)), *strides, _ptr(q_gain),
                               _ptr(k_gain), _ptr(rope_pos)), q, k, v, q_gain, k_gain, rope_pos, shape=(n, H, hd))
