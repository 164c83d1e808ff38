"""GPU: operators over drafted token trees where calls go wrong beside calls that are right: rows and trees that are
refused next to good ones, tables and stacks with holes, committed K/V that are not finite or very large, and the same rows
joined along every path.  References and tolerances are those of test_gpu_tree.py."""
import numpy as np
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree
from test_gpu_tree import (HEADS, HostPages, _attend, _batch, _cache, _close, _dev, _drafts, _host_rows, _mixed, _q, _say,
                           _shape, _upload, _want, _ws, random_parents)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ rows that are skipped beside rows that are not

@pytest.mark.parametrize("field,value", [("seq", -1), ("c", 99)])
@pytest.mark.parametrize("hd,H,trees,n,good,max_nodes", [(128, 16, 16, 16, 8, 16), (64, 55, 4, 16, 2, 16),
                                                         (64, 20, 8, 32, 4, 32), (64, 55, 4, 64, 1, 64)])
def test_skipped_rows_take_nothing_from_the_others(hd, H, trees, n, good, max_nodes, field, value):
    """Contexts of several segments; all trees fill the chip, the good ones do not.  Bit for bit what the good rows get
    without the bad ones, and what 64-bit arithmetic gets."""
    shape = _shape(hd, H)
    rng = np.random.default_rng(trees)
    made = [(1024 + 37 * (t // (trees // good)), random_parents(rng, n)) for t in range(trees)]
    at = [t // (trees // good) for t in range(trees)]  # the good trees' sequences; the others share their neighbour's
    b = _batch(rng, made, [1] * trees)
    ok = b.seq % (trees // good) == 0
    b.seq = np.array([at[t] for t in b.seq], np.int32)
    getattr(b, field)[~ok] = value
    kv, pt = _cache(shape, [(1, made[t][0] + n) for t in range(0, trees, trees // good)], 3)
    q = _q(shape, b.n, 7)
    keep = np.flatnonzero(ok)
    sel = torch.from_numpy(keep).cuda()
    _say(f"[gpu] tree attention {H} x {hd}: {good} of {trees} trees of {n} are good ({field} {value})")
    alone = _attend(shape, kv, b.take(keep), q[sel].contiguous(), max_nodes)[:len(keep)]
    got = _attend(shape, kv, b, q, max_nodes, fill=3.0, check=cdb.CDB_DEV_UNMAPPED_PAGE)[:b.n]
    assert bool((got[torch.from_numpy(~ok).cuda()] == 3.0).all())
    assert torch.equal(got[sel], alone)
    some = keep[:: max(1, len(keep) // 6)]
    want, tol = _want(shape, kv, pt, b.take(some), q[torch.from_numpy(some).cuda()])
    _close(got[torch.from_numpy(some).cuda()], want, tol)


# ------------------------------------------------------------------ trees that get no rows

@pytest.mark.parametrize("bad", [0, 1, 3])
@pytest.mark.parametrize("what", ["sequence", "negative", "twice", "length", "far", "count"])
def test_trees_without_rows_accept_nothing(what, bad):
    """A tree that cdb_tree_rows refuses, before, between and after good ones: every root is what the model says, so it
    would be accepted.  At capacity, as a captured round has it, with ids of earlier rounds behind the last row."""
    rng = np.random.default_rng(bad)
    d = _drafts(rng, [4, 3, 5, 6], 6, max_seqs=9)
    d["parent"][:] = np.arange(6) - 1
    d["tokens"][:] = 11
    if what == "twice":
        other = 2 if bad < 2 else 0
        d["seq"][bad] = d["seq"][other]
        refused = max(bad, other)
    else:
        refused = bad
        if what == "count":
            d["n_nodes"][bad] = 7
        elif what in ("length", "far"):
            d["length"][d["seq"][bad]] = -1 if what == "length" else 2 ** 31 - 2
        else:
            d["seq"][bad] = 9 if what == "sequence" else -1
    T, ws, up = 4, _ws(cdbgen.TINY, 1, 1), _upload(d)
    rows, acc = tree.TreeRows(T, 32), tree.Accepted(T, 6)
    ids, first = _dev(np.full(32, 11)), _dev(np.full(T, 11))
    _say(f"[gpu] rows and acceptance: tree {refused} is refused ({what})")
    tree.cdb_tree_rows(up.c, rows.c, ws.buf)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) == cdb.CDB_DEV_BAD_INDEX
    tree.cdb_tree_accept(up.c, rows.row0, ids, first, acc.c, ws.buf)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) in (0, cdb.CDB_DEV_BAD_INDEX)
    count = [0 if t == refused else n for t, n in enumerate((4, 3, 5, 6))]
    assert acc.count.tolist() == count and acc.next.tolist() == [11] * T
    assert acc.path.tolist() == [list(range(n)) + [-1] * (6 - n) for n in count]
    d["n_nodes"][refused] = 0
    row0, want = _host_rows(d)
    assert int(rows.n_rows) == len(want)


def test_acceptance_without_sequences():
    """Trees whose seq and len are NULL: their nodes, tokens and row0 alone count."""
    d = _drafts(np.random.default_rng(0), [4, 0, 5], 6)
    d["parent"][:] = np.arange(6) - 1
    d["tokens"][:] = 11
    up, ws, acc = _upload(d), _ws(cdbgen.TINY, 1, 1), tree.Accepted(3, 6)
    bare = tree.cdb_drafts(3, 6, 0, None, None, up.n_nodes.data_ptr(), up.parent.data_ptr(), up.tokens.data_ptr())
    tree.cdb_tree_accept(bare, _dev([0, 4, 4]), _dev(np.full(9, 11)), _dev(np.full(3, 11)), acc.c, ws.buf)
    torch.cuda.synchronize()
    assert cdb.cdb_read_device_error(ws.buf) == 0 and acc.count.tolist() == [4, 0, 5]


# ------------------------------------------------------------------ page tables and stacks with holes

@pytest.mark.parametrize("layout", [tree.KV_FULL, tree.KV_SHARED, tree.KV_FIRST_THEN_SHARED])
@pytest.mark.parametrize("S,P", [(5, 7), (60, 5), (200, 30), (300, 40)])
@pytest.mark.parametrize("where", ["table", "stack", "stack at once"])
def test_holes_in_tables_and_stacks_change_nothing(where, S, P, layout):
    """An unmapped page that a call would give back, or a hole among the pages that it would hand out: the call changes
    nothing that is mapped or free, and runs once the hole is mended.  In one workgroup and in many."""
    shape = cdbgen.TINY
    rng = np.random.default_rng(S + layout)
    caps = (S * P, S * P * shape.r_max, S * P)
    start = [rng.permutation(c).astype(np.int32) for c in caps]
    host = HostPages(shape, S, P, caps, layout, start)
    desc, ws = cdb.make_desc(shape), _ws(shape, 1, S)
    table, mapped = _dev(host.table), _dev(host.mapped)
    pools = [tree.PagePool(_dev(s), _dev([len(s)])) for s in start]

    def run(length):
        tree.cdb_map_pages(desc, table, *(p.c for p in pools), layout, _dev(length), mapped, ws.buf)
        torch.cuda.synchronize()
        return cdb.cdb_read_device_error(ws.buf)

    def same():
        n = torch.from_numpy(host.mapped).cuda()
        live = (torch.arange(P, device="cuda") < n[:, None])[:, None, :].expand(table.shape)
        assert torch.equal(table[live], torch.from_numpy(host.table).cuda()[live])
        assert (table[~live] == -1).all() and mapped.tolist() == host.mapped.tolist()
        for p, s in zip(pools, host.stacks):
            assert int(p.free_count) == len(s) and p.free_ids[:len(s)].tolist() == s

    half = rng.integers(0, 8 * P + 1, S)
    half[:2] = 16, 16 * P
    assert run(half) == host.run(half) == 0
    up = rng.random(S) < 0.5  # these grow, the others shrink
    up[:2] = True, False
    need = np.where(up, 16 * P, rng.integers(0, 9, S))
    _say(f"[gpu] map pages: {S} sequences, layout {layout}, a hole in the {where}")
    for k, planes in ((1, host.groups(1)[-1]), (0, [0])):
        stack = host.stacks[k]
        back = sum(max(0, int(m) - -(-int(n) // 16)) for m, n in zip(host.mapped, need)) * len(host.groups(k))
        more = sum(max(0, -(-int(n) // 16) - int(m)) for m, n in zip(host.mapped, need)) * len(host.groups(k))
        if where == "table" or more <= back:
            cell = (1, planes, int(host.mapped[1]) - 1)
            keep = int(host.table[1, planes[0], cell[2]])
            host.table[cell] = -1
            table[1, planes[0]:planes[-1] + 1, cell[2]] = -1
        else:
            at = len(stack) - (more - back if where == "stack" else 1)
            keep, stack[at] = stack[at], -1
            pools[k].free_ids[at] = -1
        for _ in range(2):
            assert run(need) == cdb.CDB_DEV_UNMAPPED_PAGE
            same()
        if where == "table" or more <= back:
            host.table[cell] = keep
            table[1, planes[0]:planes[-1] + 1, cell[2]] = keep
        else:
            stack[at] = keep
            pools[k].free_ids[at] = keep
    assert run(need) == host.run(need) == 0
    same()
    assert run(np.zeros(S)) == host.run(np.zeros(S)) == 0
    same()
