"""GPU: queries, keys and values of chunks of new tokens, and their attention over the paged cache, each against a plain 64-bit
implementation on the host, at the sizes, strides and masks where it can go wrong.

Tolerance of the attention.  Its output is bf16 (half a step: 2^-8 of the value).  Before that, with S the largest
sum_k |q_k K_sk| / sqrt(hd) of a row over the keys s it sees, n how many it sees and A = sum_s p_s |V_s|: the dot product
sums hd <= 128 terms in 32 bits (128 x 2^-24 = 2^-17), so a score is off by at most S x 2^-17 and every weight, over
numerator and denominator, by twice that; exp2 and the scaling add 2^-19, sums over n keys n x 2^-24 each.  bf16 queries:
weights are rounded to bf16 in the numerator, 2^-8.  fp32 queries: q is read in two bf16 parts (2^-17) and so are the
weights (2^-17).  So |error| <= 2^-8 |want| + A (2^-8 + S 2^-16 + 2^-19 + n 2^-23), and for fp32 queries
2^-8 |want| + A (2^-16 + S 2^-15 + 2^-19 + n 2^-23).

Tolerance of q, k and v.  A head's mean of squares sums hd <= 128 terms in 32 bits (half of 2^-17 after the root); root,
quotient and gains add a few 2^-24, the rotation two products, a sum and the rounded cosine and sine: with a and b the two
values that are rotated, |error| <= (|a| + |b|) 2^-17, and 2^-8 |value| where the result is bf16."""
import math
import sys

import numpy as np
import pytest
import torch

import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk

pytestmark = pytest.mark.gpu

PAGE = 16
EPS, BASE = 1e-6, 10000.0


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _desc(H, hd, layers=(1, 2, 1), r_max=3):
    return cdb.cdb_model_desc(H * hd, H, hd, 1024, 1024, *layers, r_max, 0, 0, PAGE, EPS, BASE)


class Case:
    """Chunks (rows, first position, sequence, loop), their pages scattered over a pool of one stage, and its content."""

    def __init__(self, H, hd, chunks, seed=0, stage=1, layer=1, spare_rows=0, max_pages=None, extra_pages=3):
        r = np.random.default_rng(seed)
        self.H, self.hd, self.stage, self.layer = H, hd, stage, layer
        self.desc = _desc(H, hd)
        self.chunks = [(n, p, s, c) for n, p, s, c in chunks]
        n = [x[0] for x in chunks]
        self.row0 = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        self.M = int(self.row0[-1]) + spare_rows
        S = max([x[2] for x in chunks], default=0) + 1
        longest = {}
        for nn, p, s, c in chunks:
            key = (s, self.plane(c))
            longest[key] = max(longest.get(key, 0), p + nn)
        self.P = max_pages or max(1, (max(longest.values(), default=1) + PAGE - 1) // PAGE)
        need = sum((v + PAGE - 1) // PAGE for v in longest.values())
        self.pages = need + extra_pages
        ids = r.permutation(self.pages)
        self.table = np.full((S, self.desc.r_max + 2, self.P), -1, np.int32)
        at = 0
        for (s, plane), v in longest.items():
            k = (v + PAGE - 1) // PAGE
            self.table[s, plane, :k] = ids[at:at + k]
            at += k
        layers = (self.desc.n_prelude, self.desc.n_core, self.desc.n_coda)[stage]
        g = torch.Generator().manual_seed(seed + 1)
        self.pool = torch.randn((layers, self.pages, 2, H, PAGE, hd), generator=g).to(torch.bfloat16)
        self.q = torch.randn((self.M, H * hd), generator=g) * 1.5

    def plane(self, c):
        return (0, c + 1, self.desc.r_max + 1)[self.stage]

    def device(self):
        self.d_pool, self.d_table = self.pool.cuda(), _dev(self.table)
        ptr = [None] * 3
        ptr[self.stage] = self.d_pool.data_ptr()
        count = [0] * 3
        count[self.stage] = self.pages
        self.kv = cdb.cdb_kv(*ptr, *count, self.d_table.data_ptr(), *self.table.shape[::2])
        cols = list(zip(*self.chunks)) if self.chunks else [(), (), (), ()]
        self.c = chunk.Chunks(self.M, _dev(self.row0), _dev(cols[2]), _dev(cols[1]), _dev(cols[3]))
        self.ws = chunk.ChunkWorkspace(self.desc, self.M, len(self.chunks))
        return self

    def code(self):
        return cdb.cdb_read_device_error(self.ws.buf)

    def cache(self, i, kv):
        """K or V of chunk i's context, fp64 [heads][positions][hd], and which positions are mapped."""
        n, p, s, c = self.chunks[i]
        ids = self.table[s, self.plane(c), :(p + n + PAGE - 1) // PAGE]
        x = self.pool[self.layer][torch.from_numpy(np.maximum(ids, 0)).long(), kv].double()
        x = x.permute(1, 0, 2, 3).reshape(self.H, -1, self.hd)[:, :p + n]
        return x, torch.from_numpy(np.repeat(ids >= 0, PAGE)[:p + n])

    def want(self, i, q):
        """Rows of chunk i and their tolerance, fp64 [n][d]."""
        n, p, s, c = self.chunks[i]
        r0 = int(self.row0[i])
        fp32 = q.dtype == torch.float32
        x = q[r0:r0 + n].double().view(n, self.H, self.hd).transpose(0, 1)
        (K, there), (V, _) = self.cache(i, 0), self.cache(i, 1)
        hide = (torch.arange(p + n)[None, :] > torch.arange(p, p + n)[:, None]) | ~there[None, :]
        scale = 1 / math.sqrt(self.hd)
        K0, V0 = torch.nan_to_num(K, 0, 0, 0), torch.nan_to_num(V, 0, 0, 0)  # tests that need others look at them themselves
        sc = (x @ K0.transpose(1, 2) * scale).masked_fill(hide, -math.inf)
        top = sc.amax(-1, keepdim=True).clamp(min=-1e300)
        e = torch.exp(sc - top)
        den = e.sum(-1, keepdim=True)
        den = torch.where(den == 0, 1.0, den)
        o, A = e @ V0 / den, e @ V0.abs() / den
        S = (x.abs() @ K0.abs().transpose(1, 2) * scale).masked_fill(hide, 0).amax(-1, keepdim=True)
        keys = (~hide).sum(-1)[None, :, None].double()
        if fp32:
            tol = A * (2 ** -16 + S * 2 ** -15 + 2 ** -19 + keys * 2 ** -23)
        else:
            tol = A * (2 ** -8 + S * 2 ** -16 + 2 ** -19 + keys * 2 ** -23)
        tol = tol + o.abs() * 2 ** -8
        return tuple(t.transpose(0, 1).reshape(n, -1) for t in (o, tol))

    def attend(self, dtype=torch.bfloat16, order=chunk.CDB_ORDER_ROWS, q=None, out=None, stream=None):
        q = (self.q if q is None else q).to(dtype)
        rows = self.M if order == chunk.CDB_ORDER_ROWS else (self.M + 31) // 32 * 32
        d = self.H * self.hd
        if out is None:
            out = torch.full((rows, d), 77.0, dtype=torch.bfloat16, device="cuda")
        self.d_q = q.cuda()
        chunk.cdb_chunk_attention(self.desc, self.kv, self.c.c, self.stage, self.layer, self.d_q, out, self.ws.buf,
                                  order=order, stream=stream)
        torch.cuda.synchronize()
        got = out.cpu()
        if order == chunk.CDB_ORDER_FRAGMENTS:
            got = got.view(rows // 32, d // 16, 2, 32, 8).permute(0, 3, 1, 2, 4).reshape(rows, d)[:self.M]
        return got, q

    def check(self, got, q, skip=()):
        for i, (n, p, s, c) in enumerate(self.chunks):
            if n == 0 or i in skip:
                continue
            r0 = int(self.row0[i])
            want, tol = self.want(i, q)
            err = (got[r0:r0 + n].double() - want).abs()
            worst = (err / tol.clamp(min=1e-30)).max().item()
            assert torch.isfinite(err).all() and worst <= 1, (i, self.chunks[i], worst)


def _ragged(*pairs):
    return [(n, p, i, i % 3) for i, (n, p) in enumerate(pairs)]


RAGGED = _ragged((128, 0), (129, 5), (0, 3), (1, 15), (64, 16), (33, 500), (1, 0), (200, 63), (17, 255))
SHAPES = [(4, 64), (3, 96), (2, 128), (16, 128)]


@pytest.mark.parametrize("order", [chunk.CDB_ORDER_ROWS, chunk.CDB_ORDER_FRAGMENTS])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,hd", SHAPES)
def test_attention_of_ragged_chunks(H, hd, dtype, order):
    _say(f"ragged {H} x {hd} {dtype} {order}")
    c = Case(H, hd, RAGGED, seed=1).device()
    got, q = c.attend(dtype, order)
    assert c.code() == 0
    c.check(got, q)


LENGTHS = [(1, 0), (1, 1), (1, 15), (1, 16), (2, 14), (13, 700), (31, 33), (32, 32), (1, 63), (1, 64), (64, 0), (65, 191),
           (127, 129), (128, 128), (129, 127), (1, 257), (40, 3000), (1, 5000), (300, 2500)]


@pytest.mark.parametrize("n,pos", LENGTHS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_of_one_chunk(n, pos, dtype):
    _say(f"one chunk {n} behind {pos} {dtype}")
    for H, hd in ((4, 64), (2, 128), (9, 96)):
        c = Case(H, hd, [(n, pos, 0, 2)], seed=n + pos).device()
        got, q = c.attend(dtype)
        assert c.code() == 0
        c.check(got, q)


@pytest.mark.parametrize("stage,layer", [(0, 0), (2, 0), (1, 0)])
def test_attention_in_every_stage(stage, layer):
    _say(f"stage {stage}")
    c = Case(4, 64, RAGGED, seed=2, stage=stage, layer=layer).device()
    got, q = c.attend()
    c.check(got, q)


def test_many_single_rows():
    _say("256 single rows")
    r = np.random.default_rng(3)
    c = Case(2, 128, [(1, int(p), i, i % 3) for i, p in enumerate(r.integers(0, 900, 256))], seed=3).device()
    got, q = c.attend()
    c.check(got, q)


def test_chunks_of_one_sequence_and_bits():
    """Two chunks of one sequence in one call; a chunk's bits do not depend on what the others are."""
    _say("one sequence twice")
    both = [(40, 0, 0, 1), (50, 40, 0, 1), (70, 300, 1, 0)]
    c = Case(4, 64, both, seed=4).device()
    got, q = c.attend()
    c.check(got, q)
    d = Case(4, 64, both, seed=4)
    d.pool[:, d.table[1, 1, :].tolist()] = 3.0  # the third chunk's cache
    d.device()
    other, _ = d.attend()
    assert torch.equal(other[:90], got[:90])
    assert not torch.equal(other[90:], got[90:])


def test_rows_outside_chunks_are_left():
    _say("rows outside")
    c = Case(4, 64, RAGGED, seed=5, spare_rows=37).device()
    c.row0 = c.row0 + 5  # rows 0..4 belong to nobody
    c.c = chunk.Chunks(c.M, _dev(c.row0), c.c.seq, c.c.pos0, c.c.cc)
    for dtype in (torch.bfloat16, torch.float32):
        got, q = c.attend(dtype)
        c.check(got, q)
        assert (got[:5] == 77).all() and (got[int(c.row0[-1]):] == 77).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_masked_places_hold_does_not_matter(dtype):
    """NaN and infinities behind the last position, in pages of others, in unmapped entries and in keys of later rows."""
    _say(f"masked places {dtype}")
    chunks = _ragged((3, 0), (70, 90), (1, 21), (130, 400))
    c = Case(3, 96, chunks, seed=6)
    used = torch.zeros(c.pages, PAGE, dtype=torch.bool)
    for n, p, s, loop in chunks:
        for t in range(p + n):
            used[c.table[s, loop + 1, t // PAGE], t % PAGE] = True
    for value in (math.nan, math.inf, -math.inf):
        c.pool.permute(1, 4, 0, 2, 3, 5)[~used] = value
        got, q = c.device().attend(dtype)
        c.check(got, q)
    # a value that is no number at one position of the chunk itself: rows before it are as they were
    clean = got
    n, p, s, loop = chunks[1]
    for kv in (0, 1):
        for value in (math.nan, math.inf):
            bad = 35
            d = Case(3, 96, chunks, seed=6)
            t = p + bad
            d.pool[1, d.table[s, loop + 1, t // PAGE], kv, :, t % PAGE, 5] = value
            got, q = d.device().attend(dtype)
            r0 = int(d.row0[1])
            assert torch.equal(got[:r0 + bad], clean[:r0 + bad]), (kv, value)
            assert torch.equal(got[r0 + n:], clean[r0 + n:])
            hit = got[r0 + bad:r0 + n].view(n - bad, 3, 96)
            if kv:
                assert not torch.isfinite(hit[:, :, 5]).any()
                other = [j for j in range(96) if j != 5]
                assert torch.isfinite(hit[:, :, other]).all()
            elif math.isnan(value):
                assert torch.isnan(hit).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_chunks(dtype):
    """Steps that every row of a tile sees, among them keys that are no numbers and pages that are not mapped."""
    _say(f"long chunks {dtype}")
    chunks = _ragged((1100, 333), (1024, 0))
    for H, hd in ((2, 128), (3, 96), (4, 64)):
        c = Case(H, hd, chunks, seed=8, spare_rows=3).device()
        clean, q = c.attend(dtype)
        assert c.code() == 0 and (clean[-3:] == 77).all()
        c.check(clean, q)
        p, bad = 333, 700
        for value in (math.nan, math.inf):
            d = Case(H, hd, chunks, seed=8, spare_rows=3)
            d.pool[1, d.table[0, 1, (p + bad) // PAGE], 1, :, (p + bad) % PAGE, 5] = value
            got, _ = d.device().attend(dtype)
            assert torch.equal(got[:bad], clean[:bad]) and torch.equal(got[1100:], clean[1100:])
            hit = got[bad:1100].view(1100 - bad, H, hd)
            assert not torch.isfinite(hit[:, :, 5]).any()
            assert torch.isfinite(hit[:, :, [j for j in range(hd) if j != 5]]).all()
        c.table[1, 2, 9] = -1
        c.device()
        got, q = c.attend(dtype)
        assert c.code() == cdb.CDB_DEV_UNMAPPED_PAGE
        c.check(got, q)


def test_unmapped_pages_are_left_out():
    _say("unmapped pages")
    chunks = _ragged((5, 200), (1, 700), (140, 10), (2, 30))
    c = Case(2, 128, chunks, seed=7)
    c.table[0, 1, 3] = -1
    c.table[1, 2, 40:44] = -1
    c.table[2, 3, 4] = -1
    c.table[3, 1, :2] = -1
    c.device()
    for dtype in (torch.bfloat16, torch.float32):
        got, q = c.attend(dtype)
        assert c.code() == cdb.CDB_DEV_UNMAPPED_PAGE
        c.check(got, q)
        assert (got[int(c.row0[3]):] == 0).all()  # sees nothing
    c.table[c.table == -1] = c.pages  # an id outside the pool
    c.device()
    again, _ = c.attend(torch.float32)
    assert c.code() == cdb.CDB_DEV_UNMAPPED_PAGE
    assert torch.equal(again, got)


def _bad_chunks(c):
    """(Chunks, which are refused) of every bad sequence, position and loop."""
    seq, pos, loop = (np.array(x) for x in list(zip(*c.chunks))[2:0:-1] + [list(zip(*c.chunks))[3]])
    S, R, most = c.table.shape[0], c.desc.r_max, c.P * PAGE
    for name, i, value in (("seq", 0, -1), ("seq", 1, S), ("pos", 1, -1), ("pos", 0, most), ("pos", 1, most - c.chunks[1][0] + 1),
                           ("pos", 1, 2 ** 31 - 1), ("loop", 0, -1), ("loop", 1, R)):
        a = {"seq": seq.copy(), "pos": pos.copy(), "loop": loop.copy()}
        a[name][i] = value
        yield name, i, value, chunk.Chunks(c.M, _dev(c.row0), _dev(a["seq"]), _dev(a["pos"]), _dev(a["loop"]))


def test_bad_chunks_are_skipped():
    _say("bad chunks")
    c = Case(4, 64, _ragged((7, 20), (130, 3), (2, 40)), seed=8).device()
    clean, q = c.attend()
    whole = c.c
    for name, i, value, bad in _bad_chunks(c):
        c.c = bad
        got, _ = c.attend()
        assert c.code() == cdb.CDB_DEV_BAD_INDEX, (name, value)
        a, b = int(c.row0[i]), int(c.row0[i + 1])
        assert (got[a:b] == 77).all()
        assert torch.equal(got[:a], clean[:a]) and torch.equal(got[b:], clean[b:])
    for row0 in ([0, 7, 137, 140], [-1, 7, 137, 139], [0, 137, 7, 139], [2, 1, 137, 139]):
        c.c = chunk.Chunks(c.M, _dev(row0), whole.seq, whole.pos0, whole.cc)
        got, _ = c.attend()
        assert c.code() == cdb.CDB_DEV_BAD_INDEX and (got == 77).all(), row0
    c.c = whole
    got, _ = c.attend()
    assert c.code() == 0 and torch.equal(got, clean)


def test_calls_without_rows():
    _say("no rows")
    c = Case(4, 64, [(0, 3, 0, 0), (0, 0, 1, 1)], seed=9).device()
    chunk.cdb_chunk_attention(c.desc, c.kv, c.c.c, 1, 0, torch.zeros(1, device="cuda"),
                              torch.zeros(1, dtype=torch.bfloat16, device="cuda"), c.ws.buf)
    c = Case(4, 64, [(0, 3, 0, 0), (0, 0, 1, 1)], seed=9, spare_rows=4).device()
    got, _ = c.attend()
    assert c.code() == 0 and (got == 77).all()


def test_offsets_past_32_bits():
    _say("far pages")
    H, hd, far = 16, 128, 70000  # page 70000 begins 4.6e9 values into a layer
    c = Case(H, hd, _ragged((20, 30), (1, 100)), seed=10, layer=0)
    c.desc = _desc(H, hd, (0, 1, 0))
    shift = far - c.pages
    small = c.pool[:1]
    c.pool = small
    c.device()
    big = torch.empty((1, far, 2, H, PAGE, hd), dtype=torch.bfloat16, device="cuda")
    big[0, shift:] = small[0].cuda()
    table = _dev(np.where(c.table >= 0, c.table + shift, -1))
    c.kv = cdb.cdb_kv(None, big.data_ptr(), None, 0, far, 0, table.data_ptr(), *c.table.shape[::2])
    got, q = c.attend()
    assert c.code() == 0
    c.check(got, q)
    w = Write(c, torch.bfloat16, True, seed=10)
    w.run()
    c.d_pool = big[:, shift:]
    w.check()
    del big


def test_most_rows_and_chunks():
    _say("65536 rows")
    r = np.random.default_rng(12)
    c = Case(2, 64, [(256, int(p), i, i % 3) for i, p in enumerate(r.integers(0, 60, 256))], seed=12).device()
    for dtype in (torch.bfloat16, torch.float32):
        got, q = c.attend(dtype)
        assert c.code() == 0
        c.check(got, q, skip=[i for i in range(256) if i % 37 not in (0, 36)])


def test_graphs_that_share_a_workspace():
    """Two captured calls whose segments lie in one workspace, replayed in turn."""
    _say("two graphs")
    cases = [Case(H, hd, chunks, seed=13).device() for H, hd, chunks in
             ((4, 64, _ragged((13, 700), (1, 300))), (2, 128, _ragged((3, 2000), (60, 5))))]
    ws = max((c.ws for c in cases), key=lambda w: w.buf.numel())
    clean, graphs, outs = [], [], []
    for c in cases:
        c.ws = ws
        clean.append(c.attend()[0])
        c.check(clean[-1], c.q.to(torch.bfloat16))
        outs.append(torch.zeros((c.M, c.H * c.hd), dtype=torch.bfloat16, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            chunk.cdb_chunk_attention(c.desc, c.kv, c.c.c, c.stage, c.layer, c.d_q, outs[-1], ws.buf)
    for _ in range(3):
        for g, out, want in zip(graphs, outs, clean):
            out.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.cpu(), want)


def test_another_stream_and_a_captured_call():
    """A call on a side stream; a captured call replayed with other chunks of the same capacity, twice each."""
    _say("streams and graphs")
    c = Case(4, 64, RAGGED, seed=11, spare_rows=20).device()
    clean, q = c.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, _ = c.attend(stream=side)
    assert torch.equal(got, clean)
    out = torch.full((c.M, 256), 77.0, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chunk.cdb_chunk_attention(c.desc, c.kv, c.c.c, c.stage, c.layer, c.d_q, out, c.ws.buf)
    n = len(RAGGED)
    other = np.concatenate([[0, 20], np.full(n - 1, 137)]).astype(np.int32)
    for row0 in (c.row0, other, c.row0, other):
        c.c.row0.copy_(_dev(row0))
        out.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.cpu()
        eager, _ = c.attend()
        assert torch.equal(replayed, eager)
        assert c.code() == 0


# ------------------------------------------------------------------ q, k and v

class Write:
    def __init__(self, case, dtype, norm, seed=0, gains=True, fused=True, rope=None, q_type=None, pad=0):
        g = torch.Generator().manual_seed(seed + 50)
        c = self.case = case
        M, H, hd = c.M, c.H, c.hd
        self.x = (torch.randn((M, 3, H, hd), generator=g) * 1.3).to(dtype)
        self.gains = [(1 + 0.3 * torch.randn((hd,), generator=g)).to(torch.bfloat16) if gains else None for _ in range(2)]
        self.norm, self.rope = norm, rope
        wide = torch.zeros((M, 3 * H * hd + pad), dtype=dtype)
        wide[:, :3 * H * hd] = self.x.reshape(M, -1)
        self.d_wide = wide.cuda()
        if fused:
            q, k, v = self.d_wide[:, :3 * H * hd].view(M, 3, H, hd).unbind(1) if pad == 0 else \
                self.d_wide.as_strided((M, 3, H, hd), (3 * H * hd + pad, H * hd, hd, 1)).unbind(1)
        else:
            q, k, v = (t.contiguous() for t in self.d_wide.view(M, 3, H, hd).unbind(1))
        gq, gk = (None if t is None else t.cuda() for t in self.gains)
        self.qkv = chunk.QKV(q, k, v, norm=norm, q_gain=gq, k_gain=gk, rope_pos=None if rope is None else _dev(rope))
        self.q_out = torch.full((M, H * hd), 77.0, dtype=q_type or dtype, device="cuda")

    def run(self, stream=None):
        c = self.case
        chunk.cdb_chunk_qkv(c.desc, c.kv, c.c.c, c.stage, c.layer, self.qkv.c, self.q_out, c.ws.buf, stream=stream)
        torch.cuda.synchronize()

    def turned(self, x, gain, pos):
        """fp64 [heads][hd] rotated, and |a| + |b| of what is rotated."""
        hd = x.shape[-1]
        x = x.double()
        if self.norm:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            if gain is not None:
                x = x * gain.double()
        j = torch.arange(hd // 2, dtype=torch.float64)
        a = float(pos) * BASE ** (-2 * j / hd)
        u, w = x[..., :hd // 2], x[..., hd // 2:]
        size = (u.abs() + w.abs()).repeat(1, 2)
        return torch.cat([u * a.cos() - w * a.sin(), w * a.cos() + u * a.sin()], -1), size

    def check(self, unmapped=(), skip=()):
        """unmapped: rows without a page; skip: chunks that are refused."""
        c = self.case
        pool = c.pool.clone()
        got = c.d_pool.cpu()
        q_got = self.q_out.cpu().view(c.M, c.H, c.hd)
        rows = np.zeros(c.M, bool)
        for i, (n, p, s, loop) in enumerate(c.chunks):
            if i in skip:
                continue
            for r in range(n):
                row = int(c.row0[i]) + r
                rows[row] = True
                pos = p + r
                turn = pos if self.rope is None else self.rope[row]
                want, size = self.turned(self.x[row, 0], self.gains[0], turn)
                half = 2.0 ** -8 if self.q_out.dtype == torch.bfloat16 else 0
                assert ((q_got[row].double() - want).abs() <= size * 2 ** -17 + want.abs() * half).all(), row
                if row in unmapped:
                    continue
                page = c.table[s, c.plane(loop), pos // PAGE]
                want, size = self.turned(self.x[row, 1], self.gains[1], turn)
                k = got[c.layer, page, 0, :, pos % PAGE]
                assert ((k.double() - want).abs() <= size * 2 ** -17 + want.abs() * 2 ** -8).all(), row
                assert torch.equal(got[c.layer, page, 1, :, pos % PAGE], self.x[row, 2].to(torch.bfloat16)), row
                pool[c.layer, page, :, :, pos % PAGE] = got[c.layer, page, :, :, pos % PAGE]
        assert torch.equal(pool, got)  # nothing else was written
        assert (q_got[torch.from_numpy(~rows)] == 77).all()


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("dtype,q_type", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                          (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("H,hd", SHAPES[:3])
def test_qkv_of_ragged_chunks(H, hd, dtype, q_type, norm):
    _say(f"qkv {H} x {hd} {dtype} {q_type} {norm}")
    c = Case(H, hd, _ragged((18, 0), (1, 15), (0, 3), (30, 17), (5, 4000)), seed=20, spare_rows=3).device()
    w = Write(c, dtype, norm, seed=21, q_type=q_type)
    w.run()
    assert c.code() == 0
    w.check()


@pytest.mark.parametrize("kw", [{"fused": False}, {"gains": False}, {"pad": 24}, {"pad": 8}], ids=str)
def test_qkv_strides_and_gains(kw):
    _say(f"qkv {kw}")
    c = Case(3, 96, _ragged((9, 4), (2, 70)), seed=22, stage=0, layer=0).device()
    w = Write(c, torch.bfloat16, True, seed=22, **kw)
    w.run()
    w.check()


def test_qkv_of_many_rows():
    """More rows than the form for small calls takes, other positions than the rows' own, far ones among them."""
    _say("qkv many rows")
    c = Case(1, 64, _ragged((700, 3), (1, 0), (402, 100)), seed=23).device()
    r = np.random.default_rng(23)
    rope = r.integers(-5, 200000, c.M)
    rope[:2] = 2 ** 31 - 1, 0
    w = Write(c, torch.float32, True, seed=23, rope=rope)
    w.run()
    assert c.code() == 0
    w.check()


def test_qkv_in_place():
    _say("qkv in place")
    c = Case(4, 64, _ragged((18, 0), (1, 15)), seed=24).device()
    w = Write(c, torch.float32, True, seed=24, fused=False)
    w.q_out = w.qkv.q.view(c.M, -1)
    w.run()
    w.check()


def test_qkv_unmapped_and_bad():
    _say("qkv unmapped and bad")
    chunks = _ragged((20, 10), (130, 3), (2, 40))
    c = Case(4, 64, chunks, seed=25)
    c.table[0, 1, 1] = -1
    c.table[1, 2, 2] = c.pages
    c.device()
    w = Write(c, torch.bfloat16, True, seed=25)
    w.run()
    assert c.code() == cdb.CDB_DEV_UNMAPPED_PAGE
    w.check(unmapped=[r for r in range(20) if (10 + r) // 16 == 1] + [20 + r for r in range(130) if (3 + r) // 16 == 2])
    c = Case(4, 64, _ragged((7, 20), (130, 3), (2, 40)), seed=26).device()
    for name, i, value, bad in _bad_chunks(c):
        c.device()
        c.c = bad
        w = Write(c, torch.bfloat16, True, seed=26)
        w.run()
        assert c.code() == cdb.CDB_DEV_BAD_INDEX, (name, value)
        w.check(skip=(i,))
    for row0 in ([0, 7, 137, 140], [-1, 7, 137, 139], [0, 137, 7, 139]):
        c.device()
        c.c = chunk.Chunks(c.M, _dev(row0), c.c.seq, c.c.pos0, c.c.cc)
        w = Write(c, torch.bfloat16, True, seed=26)
        w.run()
        assert c.code() == cdb.CDB_DEV_BAD_INDEX
        w.check(skip=(0, 1, 2))


def test_written_cache_is_what_attention_reads():
    """A prompt in three uneven chunks of one call each, on one captured graph each, equals the prompt as one chunk up to
    rounding, and the plain form."""
    _say("write, then attend")
    H, hd, n = 4, 64, 75
    whole = Case(H, hd, [(n, 0, 0, 1)], seed=30).device()
    w = Write(whole, torch.float32, True, seed=30)
    w.run()
    out = torch.zeros((n, H * hd), dtype=torch.bfloat16, device="cuda")
    chunk.cdb_chunk_attention(whole.desc, whole.kv, whole.c.c, 1, 1, w.q_out, out, whole.ws.buf)
    torch.cuda.synchronize()
    whole.pool = whole.d_pool.cpu()
    whole.check(out.cpu(), w.q_out.cpu())
    parts = Case(H, hd, [(n, 0, 0, 1)], seed=30).device()
    at = 0
    for size in (1, 40, 34):
        parts.c = chunk.Chunks(size, _dev([0, size]), _dev([0]), _dev([at]), _dev([1]))
        q, k, v = w.qkv.q[at:at + size], w.qkv.k[at:at + size], w.qkv.v[at:at + size]
        q_out = torch.zeros((size, H * hd), device="cuda")
        o = torch.zeros((size, H * hd), dtype=torch.bfloat16, device="cuda")
        qkv = chunk.QKV(q, k, v, norm=True, q_gain=w.qkv.q_gain, k_gain=w.qkv.k_gain)
        chunk.cdb_chunk_qkv(parts.desc, parts.kv, parts.c.c, 1, 1, qkv.c, q_out, parts.ws.buf)
        chunk.cdb_chunk_attention(parts.desc, parts.kv, parts.c.c, 1, 1, q_out, o, parts.ws.buf)
        torch.cuda.synchronize()
        assert torch.equal(q_out, w.q_out[at:at + size])
        want, tol = whole.want(0, w.q_out.cpu())
        err = (o.cpu().double() - want[at:at + size]).abs()
        assert (err <= tol[at:at + size]).all()
        at += size
    assert torch.equal(parts.d_pool, whole.d_pool)
