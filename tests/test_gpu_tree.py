"""GPU: page mapping, tree rows, tree attention, acceptance and commit, each against a plain 64-bit implementation on the
host, at the sizes and masks where it can go wrong.

Tolerance of the attention.  Its output is bf16 (half a step: 2^-8 of the value).  Before that rounding, with S the
largest sum_k |q_k K_sk| / sqrt(hd) of a row over the keys s it sees, n how many it sees and A = sum_s p_s |V_s|: q is
read to 2 x 8 bits (2^-17 relative at most: two parts, each off by half a step of the other's remainder) and the dot
product sums hd <= 128 terms in 32 bits (128 x 2^-24 = 2^-17), so a score is off by at most S x 2^-16 and every p_s, up to
the common factor that the normalisation takes out, by 2 x that (numerator and denominator); p is used to 2^-17 as well,
exp2 and the scaling add 2^-20, and sums over n keys n x 2^-24 each: |error| <= 2^-8 |want| + A (S 2^-15 + 2^-16 +
2^-19 + n 2^-23)."""
import sys

import numpy as np
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import driver as cdb_driver
from paper_2608_09444_amd import tree

pytestmark = pytest.mark.gpu

PAGE = 16


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _ws(shape, rows=256, seqs=256):
    return tree.TreeWorkspace(cdb.make_desc(shape), rows, seqs)


def random_parents(rng, n, width=4):
    """Node 0 a root; every later node below one of the `width` nodes before it, now and then a root of its own."""
    p = np.array([max(-1, j - 1 - int(rng.integers(0, width))) for j in range(n)], np.int32)
    p[:1] = -1
    return p


def ancestors(parent):
    """Masks (uint64) and depths by walking up."""
    masks, depths = [], []
    for j in range(len(parent)):
        m, d, a = 0, -1, j
        while a >= 0:
            m |= 1 << a
            d += 1
            a = int(parent[a])
        masks.append(m)
        depths.append(d)
    return np.array(masks, np.uint64), np.array(depths, np.int32)


# ------------------------------------------------------------------ page mapping

class HostPages:
    """The documented rule, one page at a time."""

    def __init__(self, shape, S, P, caps, layout, start):
        self.layout, self.R, self.P = layout, shape.r_max, P
        self.table = np.full((S, shape.r_max + 2, P), -1, np.int32)
        self.mapped = np.zeros(S, np.int32)
        self.layers = (shape.n_prelude, shape.n_core, shape.n_coda)
        self.stacks = [list(s) for s in start]
        self.arrays = [np.array(s) for s in start]  # with what stood there last above the counts
        self.caps = caps

    def groups(self, k):
        """Planes of pool k, grouped by the page they share."""
        if k != 1:
            return [[0 if k == 0 else self.R + 1]]
        if self.layout == tree.KV_FULL or self.R == 1:
            return [[p] for p in range(1, self.R + 1)]
        if self.layout == tree.KV_SHARED:
            return [list(range(1, self.R + 1))]
        return [[1], list(range(2, self.R + 1))]

    def run(self, length):
        """0, or the error code of a call that changes nothing."""
        want = [int(m) if n < 0 else (int(n) + 15) // 16 for n, m in zip(length, self.mapped)]
        if any(w > self.P for w in want):
            return cdb.CDB_DEV_BAD_INDEX
        for k in range(3):
            if not self.layers[k]:
                continue
            g = len(self.groups(k))
            back = sum(max(0, m - w) for w, m in zip(want, self.mapped)) * g
            more = sum(max(0, w - m) for w, m in zip(want, self.mapped)) * g
            if len(self.stacks[k]) + back > self.caps[k] or len(self.stacks[k]) + back < more:
                return tree.CDB_DEV_NO_PAGES
        for k in range(3):
            if not self.layers[k]:
                continue
            gone = []
            for s, w in enumerate(want):
                for p in range(w, int(self.mapped[s])):
                    for planes in self.groups(k):
                        gone.append(int(self.table[s, planes[0], p]))
                        self.table[s, planes, p] = -1
            self.stacks[k] += gone[::-1]
            self.arrays[k][:len(self.stacks[k])] = self.stacks[k]
            for s, w in enumerate(want):
                for p in range(int(self.mapped[s]), w):
                    for planes in self.groups(k):
                        self.table[s, planes, p] = self.stacks[k].pop()
        self.mapped[:] = want
        return 0


def _map_case(shape, S, P, layout, caps, steps, seed, tight=False):
    rng = np.random.default_rng(seed)
    start = [rng.permutation(c).astype(np.int32) for c in caps]
    host = HostPages(shape, S, P, caps, layout, start)
    desc = cdb.make_desc(shape)
    ws = _ws(shape, 1, S)
    table, mapped = _dev(host.table), _dev(host.mapped)
    pools = [tree.PagePool(_dev(s), _dev([len(s)])) if n else None for s, n in zip(start, host.layers)]
    codes = []
    for step in range(steps):
        n = rng.integers(0, P * PAGE + 1, S)
        n = np.where(rng.random(S) < 0.3, -1, n)
        if step == 1:
            n[:] = 0  # everything goes back
        length = n.astype(np.int32)
        code = host.run(length)
        codes.append(code)
        tree.cdb_map_pages(desc, table, *(p.c if p else None for p in pools), layout, _dev(length), mapped, ws.buf)
        torch.cuda.synchronize()
        assert cdb.cdb_read_device_error(ws.buf) == code, step
        assert (table.cpu().numpy() == host.table).all(), step
        assert (mapped.cpu().numpy() == host.mapped).all(), step
        for p, s, a in zip(pools, host.stacks, host.arrays):
            if p:
                assert int(p.free_count) == len(s) and p.free_ids.tolist() == a.tolist(), step
    return codes


@pytest.mark.parametrize("layout", [tree.KV_FULL, tree.KV_SHARED, tree.KV_FIRST_THEN_SHARED])
@pytest.mark.parametrize("S,P", [(1, 1), (5, 7), (70, 3), (300, 40)])
def test_pages_follow_the_lengths(layout, S, P):
    shape = cdbgen.TINY
    _say(f"[gpu] map pages: {S} sequences, {P} pages, layout {layout}")
    n = S * P
    codes = _map_case(shape, S, P, layout, (n, n * shape.r_max, n), 6, S + layout)
    assert codes == [0] * 6


@pytest.mark.parametrize("layout", [tree.KV_FULL, tree.KV_FIRST_THEN_SHARED])
def test_pages_of_many_sequences(layout):
    """Several sequences to a thread of every workgroup."""
    S, P, shape = 1100, 3, cdbgen.shrink(cdbgen.TINY, n_prelude=0)
    _say(f"[gpu] map pages: {S} sequences, layout {layout}")
    assert _map_case(shape, S, P, layout, (0, S * P * shape.r_max, S * P), 5, 21) == [0] * 5


@pytest.mark.parametrize("r_max", [1, 64])
def test_pages_of_models_without_prelude(r_max):
    shape = cdbgen.shrink(cdbgen.TINY, n_prelude=0, n_coda=0, r_max=r_max)
    _say(f"[gpu] map pages: r_max {r_max}, no prelude or coda")
    for layout in (tree.KV_FULL, tree.KV_SHARED, tree.KV_FIRST_THEN_SHARED):
        assert _map_case(shape, 9, 5, layout, (0, 45 * r_max, 0), 5, 3) == [0] * 5


def test_too_few_pages_change_nothing():
    _say("[gpu] map pages: pools that are sometimes too small")
    codes = _map_case(cdbgen.TINY, 12, 6, tree.KV_FULL, (40, 150, 45), 12, 8)
    assert 0 in codes and tree.CDB_DEV_NO_PAGES in codes


@pytest.mark.parametrize("what", ["length", "mapped", "count"])
def test_bad_counts_change_nothing(what):
    shape, S, P = cdbgen.TINY, 6, 4
    _say(f"[gpu] map pages: a bad {what}")
    ws = _ws(shape, 1, S)
    table = torch.full((S, shape.r_max + 2, P), -1, dtype=torch.int32, device="cuda")
    mapped = _dev(np.zeros(S))
    length = _dev([5, 17, 64, -1, 0, 33])
    pools = [tree.PagePool.full(c) for c in (24, 96, 24)]
    if what == "length":
        length[4] = 65
    elif what == "mapped":
        mapped[3] = P + 1
    else:
        pools[1].free_count.fill_(97)
    before = [t.clone() for t in (table, mapped, *(p.free_ids for p in pools), *(p.free_count for p in pools))]
    tree.cdb_map_pages(cdb.make_desc(shape), table, *(p.c for p in pools), 0, length, mapped, ws.buf)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) == cdb.CDB_DEV_BAD_INDEX
    after = (table, mapped, *(p.free_ids for p in pools), *(p.free_count for p in pools))
    assert all(torch.equal(a, b) for a, b in zip(after, before))


def test_reading_an_error_clears_that_word_alone():
    """An error code may stand in a caller's own int32; a workspace's header is cleared whole."""
    words = _dev([tree.CDB_DEV_NO_PAGES, 77, 78])
    assert cdb.cdb_read_device_error(words) == tree.CDB_DEV_NO_PAGES
    assert words.tolist() == [0, 77, 78] and cdb.cdb_read_device_error(words) == 0
    ws = torch.full((1024,), 255, dtype=torch.uint8, device="cuda")
    cdb.cdb_workspace_init(ws)
    assert ws[:8].eq(0).all() and ws[256:].eq(255).all()


@pytest.mark.parametrize("layout", [cdb_driver.KV_FULL, cdb_driver.KV_SHARED, cdb_driver.KV_FIRST_THEN_SHARED])
def test_pages_are_the_host_drivers(layout):
    """The table of the host driver after it admitted the same sequences to the same empty pools."""
    shape, lens, P = cdbgen.TINY, [40, 16, 2, 77], 6
    d = cdb_driver.Driver(4, 4, shape.r_max, 4, P, 160, 40, 40, has_prelude=True, has_coda=True, kv_layout=layout)
    for n in lens:
        d.add_sequence(n - 1, [1])
    d.next()  # plans the first call: all four are admitted
    want = d.page_table()
    _say("[gpu] map pages: as the host driver")
    table = torch.full((4, shape.r_max + 2, P), -1, dtype=torch.int32, device="cuda")
    pools = [tree.PagePool.full(c) for c in (40, 160, 40)]
    ws = _ws(shape, 1, 4)
    tree.cdb_map_pages(cdb.make_desc(shape), table, *(p.c for p in pools), layout, _dev(lens), _dev(np.zeros(4)), ws.buf)
    assert (table.cpu().numpy() == want).all()


# ------------------------------------------------------------------ rows of trees

def _drafts(rng, counts, max_nodes, max_seqs=None, vocab=1000):
    T = len(counts)
    S = max_seqs or T
    parent = np.full((T, max_nodes), 7777, np.int32)  # past a tree's nodes: not read
    for t, n in enumerate(counts):
        parent[t, :n] = random_parents(rng, n)
    seq = rng.permutation(S)[:T].astype(np.int32)
    length = rng.integers(0, 5000, S).astype(np.int32)
    tokens = rng.integers(0, vocab, (T, max_nodes)).astype(np.int32)
    return {"seq": seq, "length": length, "n_nodes": np.asarray(counts, np.int32), "parent": parent, "tokens": tokens}


def _upload(d):
    return tree.Drafts(*(_dev(d[k]) for k in ("seq", "length", "n_nodes", "parent", "tokens")))


def _host_rows(d):
    row0, out, at = [], [], 0
    for t, n in enumerate(d["n_nodes"]):
        row0.append(at)
        m, depth = ancestors(d["parent"][t, :n])
        for j in range(n):
            base = int(d["length"][d["seq"][t]])
            out.append((d["seq"][t], base + j, base, base + depth[j], d["tokens"][t, j], m[j]))
        at += int(n)
    return row0, out


NAMES = ("seq", "pos", "base", "rope_pos", "tokens", "mask")


def _check_rows(got, want, n):
    for i, name in enumerate(NAMES):
        g = getattr(got, name).cpu().numpy()[:n]
        w = np.array([r[i] for r in want[:n]], np.uint64 if name == "mask" else np.int32)
        assert (g.view(np.uint64) == w).all() if name == "mask" else (g == w).all(), name


@pytest.mark.parametrize("counts,max_nodes", [([1], 1), ([64], 64), ([0], 3), ([], 5), ([13, 0, 1, 64, 2], 64),
                                              ([1] * 256, 1), ([4] * 64, 4), ([7, 3, 33, 0, 0, 40], 50)])
def test_trees_as_rows(counts, max_nodes):
    rng = np.random.default_rng(len(counts) + max_nodes)
    d = _drafts(rng, counts, max_nodes, max_seqs=300)
    row0, want = _host_rows(d)
    n = len(want)
    out = tree.TreeRows(len(counts), n + 5)
    for name in NAMES:
        getattr(out, name).fill_(-77)
    ws = _ws(cdbgen.TINY, 1, 1)
    _say(f"[gpu] rows of {len(counts)} trees, {n} nodes")
    tree.cdb_tree_rows(_upload(d).c, out.c, ws.buf)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) == 0
    assert out.row0.tolist() == row0 and int(out.n_rows) == n
    _check_rows(out, want, n)
    for name in NAMES:  # behind the last row: left as it was
        assert (getattr(out, name)[n:] == -77).all(), name


def test_rows_of_bad_trees():
    """A bad count, sequence or length, a sequence given twice: no rows, the others as without them; a bad parent: a
    root; a tree past the capacity and those after it: no rows, row0 = -1."""
    rng = np.random.default_rng(5)
    ws = _ws(cdbgen.TINY, 1, 1)
    base = _drafts(rng, [5, 6, 7, 8, 3], 9, max_seqs=12)

    def run(d, capacity=64):
        out = tree.TreeRows(len(d["n_nodes"]), capacity)
        tree.cdb_tree_rows(_upload(d).c, out.c, ws.buf)
        torch.cuda.synchronize()
        return out, cdb.cdb_read_device_error(ws.buf)

    def without(t):
        d = {k: v.copy() for k, v in base.items()}
        d["n_nodes"][t] = 0
        return _host_rows(d)

    _say("[gpu] rows of bad trees")
    for key, t, value in (("n_nodes", 1, 10), ("n_nodes", 1, -1), ("seq", 2, 12), ("seq", 2, -1), ("seq", 3, base["seq"][0]),
                          ("length", base["seq"][4], -1), ("length", base["seq"][4], 2 ** 31 - 2)):
        d = {k: v.copy() for k, v in base.items()}
        d[key][t] = value
        out, code = run(d)
        row0, want = without(t if key != "length" else 4)
        assert code == cdb.CDB_DEV_BAD_INDEX and int(out.n_rows) == len(want) and out.row0.tolist() == row0, (key, value)
        _check_rows(out, want, len(want))
    for value in (3, 4, -2, 9):  # node 3's parent
        d = {k: v.copy() for k, v in base.items()}
        d["parent"][1, 3] = value
        out, code = run(d)
        d["parent"][1, 3] = -1
        row0, want = _host_rows(d)
        assert code == cdb.CDB_DEV_BAD_INDEX and int(out.n_rows) == len(want), value
        _check_rows(out, want, len(want))
    for capacity, fit in ((29, 5), (28, 4), (18, 3), (17, 2), (5, 1), (4, 0), (0, 0)):
        out, code = run(base, capacity)
        row0, want = _host_rows(base)
        n = int(base["n_nodes"][:fit].sum())
        assert code == (0 if fit == 5 else cdb.CDB_DEV_BAD_INDEX) and int(out.n_rows) == n, capacity
        assert out.row0.tolist() == row0[:fit] + [-1] * (5 - fit)
        _check_rows(out, want, n)


# ------------------------------------------------------------------ attention

def _shape(hd, H, **kw):
    return cdbgen.shrink(cdbgen.TINY, name=f"tree-{H}x{hd}", d=H * hd, n_heads=H, head_dim=hd, d_ff=96, n_prelude=0,
                         n_core=2, n_coda=0, **kw)


def _cache(shape, seqs, seed, spare=0):
    """Core pages of `seqs` = [(loop index, positions)]: every sequence's own plane over its positions, page ids
    shuffled.  Returns (PagedKV, page table)."""
    rng = np.random.default_rng(seed)
    P = max(1, max((n + 15) // 16 for _, n in seqs))
    pages = sum((n + 15) // 16 for _, n in seqs) + spare
    ids = rng.permutation(pages)
    pt = np.full((len(seqs), shape.r_max + 2, P), -1, np.int32)
    at = 0
    for s, (c, n) in enumerate(seqs):
        k = (n + 15) // 16
        pt[s, c + 1, :k] = ids[at:at + k]
        at += k
    kv = cdb.PagedKV(shape, len(seqs), P, 0, max(pages, 1), 0, fill="random")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kv.core.normal_(0.0, 1.0, generator=g)
    kv.page_table.copy_(torch.from_numpy(pt))
    return kv, pt


def _unfragment(out, d):
    """Fragment order -> rows."""
    n = out.numel() // d
    return out.view(n // 32, d // 16, 2, 32, 8).permute(0, 3, 1, 2, 4).reshape(n, d)


def _padded(n):
    return next(p for p in (32, 64, 128, 256) if p >= n)


class Batch:
    """Drafted rows as arrays: seq, pos, c, base, mask (uint64)."""

    def __init__(self, **kw):
        self.__dict__.update({k: np.asarray(v, np.uint64 if k == "mask" else np.int32) for k, v in kw.items()})
        self.n = len(self.seq)

    def take(self, order):
        return Batch(**{k: getattr(self, k)[order] for k in ("seq", "pos", "c", "base", "mask")})


def _batch(rng, trees, loops):
    """trees: [(base, parents)], sequence t on loop loops[t]."""
    cols = {k: [] for k in ("seq", "pos", "c", "base", "mask")}
    for t, (base, parent) in enumerate(trees):
        m, _ = ancestors(parent)
        for j in range(len(parent)):
            for k, v in zip(cols, (t, base + j, loops[t], base, m[j])):
                cols[k].append(v)
    return Batch(**cols)


def _attend(shape, kv, b, q, max_nodes, layer=1, live=None, ws=None, fill=0.0, stream=None, check=0):
    rows = cdb.Rows(np.arange(b.n), b.seq, b.pos, b.c,
                    d_n_rows=None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda"))
    see = tree.Tree(max_nodes, _dev(b.base), _dev(b.mask.view(np.int64), np.int64), _dev(b.pos))
    out = torch.full((_padded(b.n), shape.d), fill, dtype=torch.bfloat16, device="cuda")
    ws = ws or _ws(shape, b.n, 0)
    torch.cuda.synchronize()
    tree.cdb_tree_attention(cdb.make_desc(shape), kv.c, rows.c, see.c, 1, layer, q, out, ws.buf, stream=stream)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) == check
    return _unfragment(out, shape.d)


def _want(shape, kv, pt, b, q, layer=1, missing=()):
    """64-bit outputs and their bounds.  missing: page ids that are not there."""
    H, hd = shape.n_heads, shape.head_dim
    core = kv.core[layer].cpu().double()
    want, tol = torch.zeros((b.n, shape.d), dtype=torch.float64), torch.zeros((b.n, shape.d), dtype=torch.float64)
    for i in range(b.n):
        base = int(b.base[i])
        seen = list(range(base)) + [base + j for j in range(64) if int(b.mask[i]) >> j & 1]
        seen = [p for p in seen if int(pt[b.seq[i], b.c[i] + 1, p // 16]) not in missing]
        if not seen:
            continue
        pids = torch.tensor([int(pt[b.seq[i], b.c[i] + 1, p // 16]) for p in seen])
        tok = torch.tensor([p % 16 for p in seen])
        k, v = core[pids, 0, :, tok].transpose(0, 1), core[pids, 1, :, tok].transpose(0, 1)  # [H][n][hd]
        qi = q[i].cpu().double().view(H, 1, hd)
        p = torch.softmax((qi * k).sum(-1) / hd ** 0.5, -1)[..., None]
        want[i] = (p * v).sum(1).reshape(-1)
        S = ((qi * k).abs().sum(-1) / hd ** 0.5).amax(-1)[:, None]
        A = (p * v.abs()).sum(1)
        tol[i] = (want[i].abs() * 2.0 ** -8).view(-1) + \
            (A * (S * 2.0 ** -15 + 2.0 ** -16 + 2.0 ** -19 + len(seen) * 2.0 ** -23)).reshape(-1)
    return want, tol


def _close(got, want, tol, what=""):
    err = (got.double().cpu() - want).abs()
    worst = float((err / tol.clamp(min=1e-30)).max())
    assert bool((err <= tol).all()), (what, "largest error over its bound", worst, int((err / tol).argmax()) // want.shape[1])


def _q(shape, n, seed, std=1.5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 100)
    return torch.empty((n, shape.d), device="cuda").normal_(0.0, std, generator=g)


HEADS = [(64, 4), (96, 3), (128, 2)]


@pytest.mark.parametrize("hd,H", HEADS)
def test_attention_at_the_edges(hd, H):
    """Trees of 1 to 64 nodes over contexts around the page, wave and segment edges, one sequence each."""
    shape = _shape(hd, H)
    rng = np.random.default_rng(hd)
    bases = (0, 0, 1, 15, 16, 17, 31, 32, 33, 63, 100, 127, 128, 129, 255, 256, 500, 511, 512, 513, 1500, 4100)
    nodes = (1, 7, 1, 2, 15, 16, 17, 1, 5, 3, 20, 4, 2, 1, 9, 8, 13, 1, 16, 3, 33, 4)
    assert sum(nodes) <= 256 and len(bases) == len(nodes)
    trees = [(b, random_parents(rng, n)) for b, n in zip(bases, nodes)]
    loops = [t % shape.r_max for t in range(len(trees))]
    b = _batch(rng, trees, loops)
    kv, pt = _cache(shape, [(loops[t], base + len(p)) for t, (base, p) in enumerate(trees)], hd)
    q = _q(shape, b.n, 1)
    want, tol = _want(shape, kv, pt, b, q)
    for max_nodes in (64, 32, 16, 1):
        _say(f"[gpu] tree attention {H} x {hd}: {b.n} rows, max_nodes {max_nodes}")
        got = _attend(shape, kv, b, q, max_nodes)
        _close(got[:b.n], want, tol, max_nodes)
        assert bool((got[b.n:] == 0).all())


@pytest.mark.parametrize("hd,H", HEADS)
@pytest.mark.parametrize("n", [63, 64])
def test_attention_of_wide_trees(hd, H, n):
    shape = _shape(hd, H)
    rng = np.random.default_rng(n)
    trees = [(base, random_parents(rng, n, 9)) for base in (0, 41, 1003, 2500)][:256 // n]
    b = _batch(rng, trees, [0, 1, 2, 3])
    kv, pt = _cache(shape, [(t, base + n) for t, (base, p) in enumerate(trees)], n)
    q = _q(shape, b.n, 2)
    want, tol = _want(shape, kv, pt, b, q)
    for max_nodes in (64, 40):
        _say(f"[gpu] tree attention {H} x {hd}: {len(trees)} trees of {n}, max_nodes {max_nodes}")
        _close(_attend(shape, kv, b, q, max_nodes)[:b.n], want, tol)


def test_attention_of_a_wide_model_and_peaked_scores():
    """55 heads; scores up to a few hundred, as exp2 arguments far apart."""
    shape = _shape(96, 55)
    rng = np.random.default_rng(4)
    trees = [(700, random_parents(rng, 12)), (3, random_parents(rng, 12))]
    b = _batch(rng, trees, [2, 0])
    kv, pt = _cache(shape, [(2, 712), (0, 15)], 4)
    q = _q(shape, b.n, 3, std=30.0)
    want, tol = _want(shape, kv, pt, b, q)
    _say("[gpu] tree attention 55 x 96, peaked")
    _close(_attend(shape, kv, b, q, 12)[:b.n], want, tol)


def _mixed(hd=64, H=4, seed=9):
    shape = _shape(hd, H)
    rng = np.random.default_rng(seed)
    trees = [(b, random_parents(rng, n)) for b, n in ((300, 21), (0, 5), (47, 16), (1100, 9), (16, 1))]
    loops = [3, 0, 1, 2, 0]
    b = _batch(rng, trees, loops)
    kv, pt = _cache(shape, [(loops[t], base + 64) for t, (base, p) in enumerate(trees)], seed)
    return shape, trees, b, kv, pt, _q(shape, b.n, seed)


def test_rows_in_any_order_and_batch_give_the_same_bits():
    """Shuffled rows, rows interleaved over sequences, every tree alone, with any max_nodes: each row's bits stay."""
    shape, trees, b, kv, pt, q = _mixed(128, 2)
    rng = np.random.default_rng(1)
    _say("[gpu] tree attention: row order and batch")
    whole = _attend(shape, kv, b, q, 32)[:b.n]
    for order in (rng.permutation(b.n), np.argsort(np.arange(b.n) % 7, kind="stable"), np.arange(b.n)[::-1]):
        got = _attend(shape, kv, b.take(order), q[torch.from_numpy(order.copy()).cuda()].contiguous(), 32)
        assert torch.equal(got[:b.n], whole[torch.from_numpy(order.copy()).cuda()])
    for t in range(len(trees)):
        idx = np.flatnonzero(b.seq == t)
        got = _attend(shape, kv, b.take(idx), q[torch.from_numpy(idx).cuda()].contiguous(), 64)
        assert torch.equal(got[:len(idx)], whole[torch.from_numpy(idx).cuda()]), t
    one = _attend(shape, kv, b.take(np.array([5])), q[5:6].contiguous(), 1)
    assert torch.equal(one[0], whole[5])


def test_masks_of_any_shape():
    """Masks that are not a tree's: nothing but the context, nothing at all (zeros), only far bits, bit 63, all bits;
    bits on positions whose neighbours are not visible."""
    shape, trees, b, kv, pt, q = _mixed()
    m = b.mask.copy()
    first = {t: int(np.flatnonzero(b.seq == t)[0]) for t in range(5)}
    m[first[0]] = 0                    # the context alone
    m[first[0] + 1] = 1 << 63          # the context and the last position a mask reaches
    m[first[0] + 2] = 0xFFFFFFFFFFFFFFFF
    m[first[1]] = 0                    # nothing: zeros
    m[first[1] + 1] = 1 << 40          # one position, pages after an unseen page
    m[first[1] + 2] = 0x5555555555555555
    m[first[2]] = 0x8000000000000001
    m[first[4]] = 0
    b.mask = m
    want, tol = _want(shape, kv, pt, b, q)
    _say("[gpu] tree attention: masks of any shape")
    for max_nodes in (64, 16):
        got = _attend(shape, kv, b, q, max_nodes, fill=3.0)
        _close(got[:b.n], want, tol)
        assert bool((got[first[1]] == 0).all())
        assert bool((got[b.n:] == 3.0).all())


@pytest.mark.parametrize("hd,H", HEADS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_masked_positions_may_hold_anything(hd, H, value):
    """K and V of a position that a row does not see, but others of its tree do, and of positions behind the tree, do not
    reach it; those who see it get what 64-bit arithmetic gets."""
    shape, trees, b, kv, pt, q = _mixed(hd, H)
    _say(f"[gpu] tree attention {H} x {hd}: {value} in masked places")
    clean = _attend(shape, kv, b, q, 32)[:b.n]
    poison = {0: (300 + 7, 300 + 40), 1: (2, 50), 2: (47 + 15, 47 + 16), 3: (1100 + 3, 1100 + 9), 4: (17, 60)}
    for t, places in poison.items():
        for p in places:
            kv.core[1, int(pt[t, [3, 0, 1, 2, 0][t] + 1, p // 16]), :, :, p % 16] = value
    got = _attend(shape, kv, b, q, 32)[:b.n]
    hit = np.array([any(p < b.base[i] or (0 <= p - b.base[i] < 64 and int(b.mask[i]) >> int(p - b.base[i]) & 1)
                        for p in poison[int(b.seq[i])]) for i in range(b.n)])
    assert hit.any() and not hit.all()
    keep = torch.from_numpy(~hit).cuda()
    assert torch.equal(got[keep], clean[keep])
    # a NaN or infinite V that a row sees makes its output not finite, in every dim
    assert not bool(torch.isfinite(got[~keep]).any())


def test_values_alone_that_are_not_finite():
    """Finite K, infinite V in one dim of one drafted position: only that dim of the rows that see it."""
    shape, trees, b, kv, pt, q = _mixed(64, 4)
    clean = _attend(shape, kv, b, q, 32)[:b.n]
    p = 300 + 4
    kv.core[1, int(pt[0, 4, p // 16]), 1, 2, p % 16, 9] = float("inf")
    _say("[gpu] tree attention: one infinite value")
    got = _attend(shape, kv, b, q, 32)[:b.n]
    sees = torch.tensor([int(b.seq[i]) == 0 and int(b.mask[i]) >> 4 & 1 == 1 for i in range(b.n)]).cuda()
    dim = 2 * 64 + 9
    assert bool((got[sees][:, dim] == float("inf")).all()) and bool(sees.any())
    got[sees, dim] = clean[sees, dim]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("live", [0, 1, 20, 21, 22, 40, 52])
def test_device_row_count(live):
    shape, trees, b, kv, pt, q = _mixed()
    _say(f"[gpu] tree attention: {live} of {b.n} rows")
    whole = _attend(shape, kv, b, q, 16)
    got = _attend(shape, kv, b, q, 16, live=live, fill=3.0)
    n = min(live, b.n)
    assert torch.equal(got[:n], whole[:n]) and bool((got[n:] == 3.0).all())


def test_pages_and_indices_out_of_range():
    """An unmapped page is left out; a row of a bad sequence, loop, base or mask is skipped; the others keep their bits."""
    shape, trees, b, kv, pt, q = _mixed()
    whole = _attend(shape, kv, b, q, 16)[:b.n]
    _say("[gpu] tree attention: bad pages and indices")
    gone = int(pt[0, 4, 5])
    for bad in (-1, kv.core.shape[1]):
        kv.page_table[0, 4, 5] = bad
        got = _attend(shape, kv, b, q, 16, check=cdb.CDB_DEV_UNMAPPED_PAGE)[:b.n]
        want, tol = _want(shape, kv, pt, b, q, missing=(gone,))
        _close(got, want, tol)
        other = torch.from_numpy(b.seq != 0).cuda()
        assert torch.equal(got[other], whole[other])
    kv.page_table.copy_(torch.from_numpy(pt))
    cap = pt.shape[2] * PAGE
    for field, value in (("seq", 5), ("seq", -1), ("c", shape.r_max), ("c", -1), ("base", -1), ("base", cap + 1),
                         ("base", cap - 62), ("base", 2 ** 31 - 1)):
        rows = b.take(np.arange(b.n))
        i = 8
        getattr(rows, field)[i] = value
        if field == "base":
            rows.mask[i] = 1 << 62
        got = _attend(shape, kv, rows, q, 16, check=cdb.CDB_DEV_UNMAPPED_PAGE, fill=3.0)[:b.n]
        assert bool((got[i] == 3.0).all()), (field, value)
        keep = torch.arange(b.n, device="cuda") != i
        assert torch.equal(got[keep], whole[keep]), (field, value)


def test_attention_captured_and_on_another_stream():
    """A graph replayed between eager calls of another size on the same workspace, and a call on a side stream."""
    shape, trees, b, kv, pt, q = _mixed(128, 2)
    ws = _ws(shape, 256, 0)
    want = _attend(shape, kv, b, q, 32, ws=ws)[:b.n]
    rows = cdb.Rows(np.arange(b.n), b.seq, b.pos, b.c)
    see = tree.Tree(32, _dev(b.base), _dev(b.mask.view(np.int64), np.int64), _dev(b.pos))
    out = torch.zeros((_padded(b.n), shape.d), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    _say("[gpu] tree attention: captured")
    with torch.cuda.graph(graph, stream=side):
        tree.cdb_tree_attention(cdb.make_desc(shape), kv.c, rows.c, see.c, 1, 1, q, out, ws.buf, stream=side)
    few = b.take(np.arange(7))
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(_unfragment(out, shape.d)[:b.n], want)
        got = _attend(shape, kv, few, q[:7].contiguous(), 16, ws=ws)
        assert torch.equal(got[:7], want[:7])
    assert torch.equal(_attend(shape, kv, b, q, 32, ws=ws, stream=side)[:b.n], want)


def _graph(call):
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    return graph


def test_graphs_that_share_a_workspace():
    """Page mapping up and down and attention of contexts with and without records, each in a graph of its own, replayed in
    turn with eager calls between."""
    shape = _shape(128, 4)
    rng = np.random.default_rng(13)
    kv, pt = _cache(shape, [(0, 2600), (1, 300), (2, 64)], 41)
    ws, desc = _ws(shape, 64, 40), cdb.make_desc(shape)
    calls, outs, wants = [], [], []
    for trees, loops in (([(2500, random_parents(rng, 9))], [0]), ([(7, [-1]), (250, random_parents(rng, 13))], [0, 1])):
        b = _batch(rng, trees, loops)
        rows = cdb.Rows(np.arange(b.n), b.seq, b.pos, b.c)
        see = tree.Tree(16, _dev(b.base), _dev(b.mask.view(np.int64), np.int64), _dev(b.pos))
        q, out = _q(shape, b.n, 51 + b.n), torch.zeros((32, shape.d), dtype=torch.bfloat16, device="cuda")
        calls.append(lambda rows=rows, see=see, q=q, out=out: tree.cdb_tree_attention(desc, kv.c, rows.c, see.c, 1, 1, q,
                                                                                       out, ws.buf))
        outs.append(out)
    table = torch.full((40, shape.r_max + 2, 30), -1, dtype=torch.int32, device="cuda")
    mapped, pool = _dev(np.zeros(40)), tree.PagePool.full(40 * 30 * shape.r_max)
    low = rng.integers(0, 130, 40)
    for need in (_dev(low + rng.integers(0, 350, 40)), _dev(low)):
        calls.append(lambda need=need: tree.cdb_map_pages(desc, table, None, pool.c, None, 0, need, mapped, ws.buf))
    for k, call in enumerate(calls):
        call()
        torch.cuda.synchronize()
        wants.append(outs[k].clone() if k < 2 else None)
    # every sequence grows, then is cut back: each state repeats, with its stack
    states = {}
    graphs = [_graph(call) for call in calls]
    _say("[gpu] four graphs of one workspace")
    for turn in range(4):
        for k in (2, 0, 3, 1):
            (graphs[k].replay if turn % 2 else calls[k])()
            torch.cuda.synchronize()
            if k < 2:
                assert torch.equal(outs[k], wants[k]), (turn, k)
                outs[k].zero_()
            else:
                now = (table.clone(), mapped.clone(), pool.free_count.clone(), pool.free_ids[:int(pool.free_count)].clone())
                for a, b in zip(now, states.setdefault(k, now)):
                    assert torch.equal(a, b), (turn, k)
    assert cdb.cdb_read_device_error(ws.buf) == 0
    del graphs


def test_a_long_context_with_pages_past_32_bit_offsets():
    """Pages whose byte offsets in the pool pass 2^32, and 20011 positions."""
    shape = _shape(128, 16)
    rng = np.random.default_rng(2)
    base, n = 20011, 10
    spare = (1 << 32) // (2 * 16 * 16 * 128 * 2) + 8
    b = _batch(rng, [(base, random_parents(rng, n))], [1])
    kv, pt = _cache(shape, [(1, base + n)], 6, spare=spare)
    hi = np.sort(pt[0, 2])[::-1].copy()
    assert int(hi[0]) * 2 * 16 * 16 * 128 * 2 > 1 << 32
    q = _q(shape, n, 5)
    H = 16
    _say("[gpu] tree attention: 20011 positions, pages past 4 GiB")
    got = _attend(shape, kv, b, q, 16)[:n]
    core = kv.core[1, torch.from_numpy(pt[0, 2].astype(np.int64)).cuda()].cpu()
    k, v = (core[:, t].permute(1, 0, 2, 3).reshape(H, -1, 128)[:, :base + n].double() for t in (0, 1))
    qd = q.cpu().double().view(n, H, 128)
    for i in range(n):
        sc = (k * qd[i][:, None]).sum(-1) / 128 ** 0.5
        hide = torch.tensor([not int(b.mask[i]) >> j & 1 for j in range(n)])
        sc[:, base:][:, hide] = -float("inf")
        p = torch.softmax(sc, -1)[..., None]
        want = (p * v).sum(1)
        S = ((k * qd[i][:, None]).abs().sum(-1) / 128 ** 0.5).amax(-1)[:, None]
        tol = want.abs() * 2.0 ** -8 + (p * v.abs()).sum(1) * (S * 2.0 ** -15 + 2.0 ** -16 + 2.0 ** -19 + (base + n) * 2.0 ** -23)
        assert bool(((got[i].cpu().double().view(H, 128) - want).abs() <= tol).all()), i


# ------------------------------------------------------------------ acceptance

def _host_accept(d, says, first):
    T, N = d["parent"].shape
    path, count, nxt = np.full((T, N), -1, np.int32), np.zeros(T, np.int32), first.copy()
    for t in range(T):
        at = -1
        while True:
            kids = [j for j in range(d["n_nodes"][t]) if d["parent"][t, j] == at and j > at and d["tokens"][t, j] == nxt[t]]
            if not kids:
                break
            at = kids[0]
            path[t, count[t]] = at
            count[t] += 1
            nxt[t] = says[t, at]
    return path, count, nxt


def _accept_case(rng, counts, max_nodes, vocab):
    """A small vocabulary: tokens agree often, and siblings often hold the same token."""
    d = _drafts(rng, counts, max_nodes, vocab=vocab)
    says = rng.integers(0, vocab, d["parent"].shape).astype(np.int32)
    first = rng.integers(0, vocab, len(counts)).astype(np.int32)
    return d, says, first


def _accept(d, says, first, row0=None, n_rows=None):
    T, N = d["parent"].shape
    n = np.clip(d["n_nodes"], 0, N)
    starts = np.cumsum(n) - n
    ids = np.concatenate([says[t, :n[t]] for t in range(T)] + [np.zeros(1, np.int32)])[:-1]
    ids = ids if n_rows is None else ids[:n_rows]
    out = tree.Accepted(T, N)
    for x in (out.path, out.count, out.next):
        x.fill_(77)
    ws = _ws(cdbgen.TINY, 1, 1)
    tree.cdb_tree_accept(_upload(d).c, _dev(starts if row0 is None else row0), _dev(ids), _dev(first), out.c, ws.buf)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (out.path, out.count, out.next)], cdb.cdb_read_device_error(ws.buf)


@pytest.mark.parametrize("counts,max_nodes,vocab", [([1], 1, 1), ([1], 1, 2), ([64], 64, 1), ([64, 0, 63, 1], 64, 2),
                                                    ([4] * 64, 4, 2), ([1] * 256, 1, 2), ([9, 30, 17], 30, 3)])
def test_acceptance(counts, max_nodes, vocab):
    rng = np.random.default_rng(len(counts) + vocab)
    _say(f"[gpu] accept: {len(counts)} trees of up to {max_nodes}, {vocab} tokens")
    for _ in range(4):
        d, says, first = _accept_case(rng, counts, max_nodes, vocab)
        got, code = _accept(d, says, first)
        assert code == 0
        for g, w in zip(got, _host_accept(d, says, first)):
            assert (g == w).all()


def test_acceptance_of_chains_to_the_end():
    """64 nodes below one another, all as the model says, and one wrong token at every place."""
    d = _drafts(np.random.default_rng(1), [64] * 65, 64)
    d["parent"][:] = np.arange(64) - 1
    says = np.concatenate([d["tokens"][:, 1:], np.full((65, 1), 5, np.int32)], 1)
    first = d["tokens"][:, 0].copy()
    for t in range(64):
        d["tokens"][t, t] = 100000
    (path, count, nxt), code = _accept(d, says, first)
    assert code == 0 and count.tolist() == list(range(65)) and nxt[64] == 5
    assert (path[64] == np.arange(64)).all() and (path[10] == np.where(np.arange(64) < 10, np.arange(64), -1)).all()


def test_acceptance_of_bad_trees():
    """Trees without rows accept nothing; nodes whose rows are out of range, or whose parents are not earlier nodes, are
    not reached; a bad count is no nodes."""
    rng = np.random.default_rng(2)
    d, says, first = _accept_case(rng, [8, 8, 8, 8], 8, 1)
    d["parent"][:] = np.arange(8) - 1
    _say("[gpu] accept: bad trees")
    (path, count, nxt), code = _accept(d, says, first, row0=[0, -1, 16, 24], n_rows=29)
    assert code == cdb.CDB_DEV_BAD_INDEX and count.tolist() == [8, 0, 8, 5] and (path[1] == -1).all()
    e = {k: v.copy() for k, v in d.items()}
    e["parent"][0, 3], e["parent"][1, 3], e["parent"][2, 3] = 3, 7, -5
    e["n_nodes"][3] = 9
    (path, count, nxt), code = _accept(e, says, first, row0=[0, 8, 16, 24])
    assert count.tolist() == [3, 3, 3, 0]


# ------------------------------------------------------------------ commit

def _commit_setup(shape, counts, max_nodes, layout, seed, lo=0, hi=200):
    """A cache with every plane mapped over each sequence's length + nodes, random paths."""
    rng = np.random.default_rng(seed)
    T = len(counts)
    seq = rng.permutation(T + 2)[:T].astype(np.int32)
    length = rng.integers(lo, hi, T + 2).astype(np.int32)
    P = int((length.max() + max_nodes + 15) // 16)
    n = (T + 2) * P
    ws = _ws(shape, 1, T + 2)
    kv = cdb.PagedKV(shape, T + 2, P, n, n * shape.r_max, n, fill="random")
    pools = [tree.PagePool(_dev(rng.permutation(c)), _dev([c])) if k else None
             for c, k in ((n, shape.n_prelude), (n * shape.r_max, shape.n_core), (n, shape.n_coda))]
    tree.cdb_map_pages(cdb.make_desc(shape), kv.page_table, *(p.c if p else None for p in pools), layout,
                       _dev(length + max_nodes), _dev(np.zeros(T + 2)), ws.buf)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for x in (kv.pre, kv.core, kv.coda):
        x.normal_(0.0, 1.0, generator=g)
    path = np.full((T, max_nodes), -1, np.int32)
    for t, c in enumerate(counts):
        path[t, :c] = np.sort(rng.permutation(max_nodes)[:c])
    return kv, seq, length, path, np.asarray(counts, np.int32), ws


def _host_commit(shape, pools, pt, seq, length, path, count):
    """pools: [(pool, planes)], on the host; a page's moves once, whatever planes map it."""
    for pool, planes in pools:
        for t in range(len(seq)):
            base, moved = int(length[seq[t]]), set()
            for pl in planes:
                ids = pt[seq[t], pl]
                key = tuple(ids[base // 16:(base + 64) // 16 + 1])
                if key in moved:
                    continue
                moved.add(key)
                for i in range(count[t]):
                    s, e = base + int(path[t, i]), base + i
                    pool[:, ids[e // 16], :, :, e % 16] = pool[:, ids[s // 16], :, :, s % 16].clone()


def _run_commit(shape, kv, seq, length, path, count, ws, max_nodes):
    T = len(seq)
    acc = tree.Accepted(T, max_nodes)
    acc.path.copy_(torch.from_numpy(path))
    acc.count.copy_(torch.from_numpy(count))
    z = np.zeros((T, max_nodes), np.int32)
    d = tree.Drafts(_dev(seq), _dev(length), _dev(np.zeros(T)), _dev(z), _dev(z))
    tree.cdb_tree_commit(cdb.make_desc(shape), kv.c, d.c, acc.c, ws.buf)
    torch.cuda.synchronize()
    return cdb.cdb_read_device_error(ws.buf)


def _stages(shape, kv):
    R = shape.r_max
    return [(p, planes) for p, planes, n in ((kv.pre, [0], shape.n_prelude), (kv.core, range(1, R + 1), shape.n_core),
                                             (kv.coda, [R + 1], shape.n_coda)) if n]


COMMITS = [([1], 1), ([3], 5), ([0], 4), ([64], 64), ([9, 0, 64, 40, 1], 64), ([4] * 40, 4), ([10, 11, 12, 13], 40)]


@pytest.mark.parametrize("layout", [tree.KV_FULL, tree.KV_SHARED, tree.KV_FIRST_THEN_SHARED])
@pytest.mark.parametrize("counts,max_nodes", COMMITS)
def test_commit_moves_the_path(layout, counts, max_nodes):
    shape = cdbgen.shrink(cdbgen.TINY, n_core=3) if len(counts) < 3 else cdbgen.shrink(cdbgen.TINY, n_prelude=0, n_coda=0)
    kv, seq, length, path, count, ws = _commit_setup(shape, counts, max_nodes, layout, len(counts) + max_nodes)
    host = [(p.cpu().clone(), planes) for p, planes in _stages(shape, kv)]
    _host_commit(shape, host, kv.page_table.cpu().numpy(), seq, length, path, count)
    _say(f"[gpu] commit: {len(counts)} trees of up to {max_nodes}, layout {layout}")
    assert _run_commit(shape, kv, seq, length, path, count, ws, max_nodes) == 0
    for (got, _), (want, _) in zip(_stages(shape, kv), host):
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("hd,H", [(96, 55), (128, 16)])
def test_commit_of_wide_models(hd, H):
    shape = _shape(hd, H)
    kv, seq, length, path, count, ws = _commit_setup(shape, [20, 5, 33], 50, tree.KV_FULL, hd)
    host = [(p.cpu().clone(), planes) for p, planes in _stages(shape, kv)]
    _host_commit(shape, host, kv.page_table.cpu().numpy(), seq, length, path, count)
    _say(f"[gpu] commit {H} x {hd}")
    assert _run_commit(shape, kv, seq, length, path, count, ws, 50) == 0
    assert torch.equal(kv.core.cpu(), host[0][0])


def test_commit_of_many_layers_and_trees():
    """1088 (layer, plane, tree) triples of 320 columns: one workgroup each."""
    shape = _shape(64, 20)
    shape = cdbgen.shrink(shape, n_core=16)
    counts = [int(c) for c in np.random.default_rng(3).integers(0, 9, 17)]
    kv, seq, length, path, count, ws = _commit_setup(shape, counts, 8, tree.KV_FULL, 31, hi=20)
    host = [(kv.core.cpu().clone(), range(1, shape.r_max + 1))]
    _host_commit(shape, host, kv.page_table.cpu().numpy(), seq, length, path, count)
    _say("[gpu] commit: many layers and trees")
    assert _run_commit(shape, kv, seq, length, path, count, ws, 8) == 0
    assert torch.equal(kv.core.cpu(), host[0][0])


def test_commit_refuses_what_it_cannot_move():
    """Bad paths, sequences and planes leave their own pages alone, and the other trees move."""
    shape, N = cdbgen.shrink(cdbgen.TINY, n_prelude=0, n_coda=0, n_core=1), 30
    kv, seq, length, path, count, ws = _commit_setup(shape, [9, 12, 7], N, tree.KV_FULL, 77, lo=20, hi=40)
    pool, pt = kv.core.clone(), kv.page_table.cpu().numpy().copy()
    _say("[gpu] commit: refusals")

    def run(code, moves, table=None, **kw):
        a = {"seq": seq.copy(), "length": length.copy(), "path": path.copy(), "count": count.copy()}
        for k, (at, v) in kw.items():
            a[k][at] = v
        kv.core.copy_(pool)
        kv.page_table.copy_(torch.from_numpy(pt if table is None else table))
        host = pool.cpu().clone()
        for t in moves:
            _host_commit(shape, [(host, range(1, shape.r_max + 1))], pt, seq[t:t + 1], length, path[t:t + 1], count[t:t + 1])
        assert _run_commit(shape, kv, a["seq"], a["length"], a["path"], a["count"], ws, N) == code, kw
        assert torch.equal(kv.core.cpu(), host), kw

    B = cdb.CDB_DEV_BAD_INDEX
    run(0, [0, 1, 2])
    run(B, [0, 2], count=(1, N + 1))
    run(B, [0, 2], count=(1, -1))
    run(B, [0, 2], seq=(1, 5))
    run(B, [0, 2], seq=(1, -1))
    run(B, [0, 2], seq=(1, seq[0]))
    run(B, [0, 2], path=((1, 3), path[1, 2]))
    run(B, [0, 2], path=((1, 11), N))
    run(B, [0, 2], path=((1, 0), -1))
    run(B, [0, 2], length=(seq[1], pt.shape[2] * 16 - 3))
    run(B, [0, 2], length=(seq[1], -1))
    # one page unmapped in every plane of a tree; planes 1 and 2 on one page of several
    page = (int(length[seq[1]]) + int(path[1, 11])) // 16
    t2 = pt.copy()
    t2[seq[1], 1:shape.r_max + 1, page] = -1
    run(cdb.CDB_DEV_UNMAPPED_PAGE, [0, 2], table=t2)
    t2 = pt.copy()
    t2[seq[1], 1:shape.r_max + 1, page] = t2[seq[1], 1, page]
    run(B, [0, 2], table=t2)
