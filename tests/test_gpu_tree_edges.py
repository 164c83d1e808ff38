"""GPU: operators over drafted token trees where calls go wrong beside calls that are right: rows and trees that are
refused next to good ones, tables and stacks with holes, committed K/V that are not finite or very large, and the same rows
joined along every path.  References and tolerances are those of test_gpu_tree.py."""
import numpy as np
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree
from test_gpu_tree import (HEADS, HostPages, _attend, _batch, _cache, _close, _dev, _drafts, _graph, _host_rows, _mixed, _q,
                           _say, _shape, _upload, _want, _ws, random_parents)

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


@pytest.mark.parametrize("S,P", [(60, 5), (300, 40)])
def test_captured_mappings_and_holes(S, P):
    """Growing and cutting back in graphs, replayed in turn; now and then a hole, mended before the next replay."""
    shape, layout = cdbgen.TINY, tree.KV_FULL
    rng = np.random.default_rng(S)
    caps = (S * P, S * P * shape.r_max, S * P)
    start = [rng.permutation(c).astype(np.int32) for c in caps]
    host = HostPages(shape, S, P, caps, layout, start)
    desc, ws = cdb.make_desc(shape), _ws(shape, 1, S)
    table, mapped = _dev(host.table), _dev(host.mapped)
    pools = [tree.PagePool(_dev(s), _dev([len(s)])) for s in start]
    needs = [np.where(rng.random(S) < 0.1, -1, rng.integers(16, 16 * P + 1, S)), rng.integers(0, 16 * P + 1, S)]
    needs[0][0], needs[1][0] = 16 * P, 0
    up = [_dev(n) for n in needs]
    calls = [lambda n=n: tree.cdb_map_pages(desc, table, *(p.c for p in pools), layout, n, mapped, ws.buf) for n in up]
    graphs = [_graph(call) for call in calls]
    _say(f"[gpu] captured mappings of {S} sequences")
    for turn in range(8):
        k = turn % 2
        cell = (0, 2, P - 1)
        if k == 1 and turn % 4 == 3:  # the first sequence gives everything back
            keep = int(host.table[cell])
            table[cell] = -1
            graphs[k].replay()
            torch.cuda.synchronize()
            assert cdb.cdb_read_device_error(ws.buf) == cdb.CDB_DEV_UNMAPPED_PAGE and mapped.tolist() == host.mapped.tolist()
            table[cell] = keep
        (calls[k] if turn in (2, 5) else graphs[k].replay)()
        torch.cuda.synchronize()
        assert host.run(needs[k]) == 0 and cdb.cdb_read_device_error(ws.buf) == 0
        assert (table.cpu().numpy() == host.table).all() and mapped.tolist() == host.mapped.tolist(), turn
        for p, s in zip(pools, host.stacks):
            assert int(p.free_count) == len(s) and p.free_ids[:len(s)].tolist() == s, turn
    del graphs


# ------------------------------------------------------------------ committed K/V that are not finite, or large

def _place(pt, t, position, loop):
    """(page id, token) of a position of sequence t in the loop's plane."""
    return int(pt[t, loop + 1, position // 16]), position % 16


LOOPS = (3, 0, 1, 2, 0)  # of _mixed's trees


@pytest.mark.parametrize("hd,H", HEADS)
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_committed_values_that_are_not_finite(hd, H, value):
    """V of one dim of a committed position, in contexts of one segment and of several: that dim of the tree's rows becomes
    what 64-bit arithmetic gets, everything else keeps its bits."""
    shape, trees, b, kv, pt, q = _mixed(hd, H)
    clean = _attend(shape, kv, b, q, 32)[:b.n]
    dim = 1 * hd + 9
    for t, position in ((0, 130), (2, 46), (3, 1050), (3, 17), (4, 3)):
        page, tok = _place(pt, t, position, LOOPS[t])
        before = kv.core[1, page, 1, 1, tok, 9].clone()
        kv.core[1, page, 1, 1, tok, 9] = value
        _say(f"[gpu] tree attention {H} x {hd}: V {value} at committed position {position}")
        got = _attend(shape, kv, b, q, 32)[:b.n]
        kv.core[1, page, 1, 1, tok, 9] = before
        mine = torch.from_numpy(b.seq == t).cuda()
        if value == value:
            assert bool((got[mine, dim] == value).all()), (t, got[mine, dim])
        else:
            assert bool(got[mine, dim].isnan().all())
        got[mine, dim] = clean[mine, dim]
        assert torch.equal(got, clean)


@pytest.mark.parametrize("max_nodes", [16, 32, 64])
def test_committed_values_that_are_not_finite_in_full_batches(max_nodes):
    """Segments joined in registers (144 tiles and heads or more): the same."""
    shape = _shape(128, 16)
    rng = np.random.default_rng(4)
    made = [(1030 + 5 * t, random_parents(rng, 3)) for t in range(9)]
    b = _batch(rng, made, [0] * 9)
    kv, pt = _cache(shape, [(0, base + 3) for base, _ in made], 8)
    q = _q(shape, b.n, 8)
    clean = _attend(shape, kv, b, q, max_nodes)[:b.n]
    for t in (0, 4, 8):
        page, tok = _place(pt, t, 500 + t, 0)
        kv.core[1, page, 1, 5, tok, 77] = float("inf")
    _say(f"[gpu] tree attention 16 x 128: infinite committed V, 9 trees, max_nodes {max_nodes}")
    got = _attend(shape, kv, b, q, max_nodes)[:b.n]
    mine, dim = torch.from_numpy(b.seq % 4 == 0).cuda(), 5 * 128 + 77
    assert bool((got[mine, dim] == float("inf")).all())
    got[mine, dim] = clean[mine, dim]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("hd,H", HEADS)
def test_committed_keys_that_are_not_finite(hd, H):
    """One dim of one committed K is -inf: where q is positive there the key has no weight, where it is negative its score
    is +inf and the head's output NaN; other heads and trees keep their bits."""
    shape, trees, b, kv, pt, q = _mixed(hd, H)
    _say(f"[gpu] tree attention {H} x {hd}: K -inf at a committed position")
    clean, signs = _attend(shape, kv, b, q, 32)[:b.n], set()
    for t, position in ((0, 131), (3, 1049), (3, 5), (4, 15)):
        page, tok = _place(pt, t, position, LOOPS[t])
        before = kv.core[1, page, 0, 1, tok].clone()
        rows = np.flatnonzero(b.seq == t)
        sel = torch.from_numpy(rows).cuda()
        kv.core[1, page, 0, 1, tok, 3] = -float("inf")
        got = _attend(shape, kv, b, q, 32)[:b.n]
        plus = q[sel][:, hd + 3].cpu() > 0
        signs |= set(plus.tolist())
        for i, r in enumerate(rows):
            mine = got[r].cpu().double().view(H, hd)[1]
            if not plus[i]:
                assert bool(mine.isnan().all()), (t, position, r)
                continue
            core = kv.core[1].cpu().double()
            seen = list(range(int(b.base[r]))) + [int(b.base[r]) + j for j in range(64) if int(b.mask[r]) >> j & 1]
            seen.remove(position)
            ids = torch.tensor([int(pt[t, LOOPS[t] + 1, p // 16]) for p in seen])
            at = torch.tensor([p % 16 for p in seen])
            k, v = core[ids, 0, 1, at], core[ids, 1, 1, at]
            qi = q[r].cpu().double().view(H, hd)[1]
            p = torch.softmax((k * qi).sum(-1) / hd ** 0.5, -1)
            w = (p[:, None] * v).sum(0)
            S = ((k * qi).abs().sum(-1) / hd ** 0.5).max()
            bound = w.abs() * 2.0 ** -8 + (p[:, None] * v.abs()).sum(0) * \
                (S * 2.0 ** -15 + 2.0 ** -16 + 2.0 ** -19 + len(seen) * 2.0 ** -23)
            assert bool(((mine - w).abs() <= bound).all()), (t, position, r)
        kv.core[1, page, 0, 1, tok] = before
        got.view(b.n, H, hd)[sel, 1] = clean.view(b.n, H, hd)[sel, 1]
        assert torch.equal(got, clean)
    assert signs == {True, False}


def _one_sequence(hd, H, base, k, v, q):
    """One row over `base` committed positions and its own, all with these K and V."""
    shape = _shape(hd, H)
    b = _batch(np.random.default_rng(0), [(base, np.array([-1], np.int32))], [0])
    kv, pt = _cache(shape, [(0, base + 1)], 1)
    kv.core[1, :, 0] = k
    kv.core[1, :, 1] = v
    return shape, b, kv, torch.full((1, shape.d), q, device="cuda")


@pytest.mark.parametrize("hd,H", HEADS)
@pytest.mark.parametrize("base", [0, 1, 40, 1200])
def test_scores_and_sums_at_the_ends_of_the_range(hd, H, base):
    """Equal keys, so the output is V itself (each weight the same; off by the sum of base + 1 weights in 32 bits, and half a
    step): scores of about -1e33, and V of 2e38, whose plain sum has no 32-bit value.  Nothing but scores of -inf: NaN."""
    n = base + 1
    for k, v, q in ((-2.0 ** 50, 1.25, 2.0 ** 57), (0.0, 2.0 ** 127 * 1.25, 1.0), (2.0 ** 50, -3.0, -(2.0 ** 57))):
        shape, b, kv, qq = _one_sequence(hd, H, base, k, v, q)
        _say(f"[gpu] tree attention {H} x {hd}: {n} keys of {k}, values of {v}")
        got = _attend(shape, kv, b, qq, 1)[:1].double().cpu()
        assert bool(((got - v).abs() <= abs(v) * (2.0 ** -8 + n * 2.0 ** -22)).all()), got
    shape, b, kv, qq = _one_sequence(hd, H, base, -float("inf"), 1.0, 1.0)
    assert bool(_attend(shape, kv, b, qq, 1)[0].isnan().all())


# ------------------------------------------------------------------ one row, every way its segments are joined

@pytest.mark.parametrize("hd,H", [(64, 16), (96, 16), (128, 16)])
@pytest.mark.parametrize("max_nodes,n", [(16, 13), (32, 25), (64, 28)])
def test_records_and_registers_give_the_same_bits(hd, H, max_nodes, n):
    """Trees over several segments, in a batch of at least 144 (tile, head) pairs, whose segments are joined in registers, and
    alone, where they go through records."""
    shape = _shape(hd, H)
    rng = np.random.default_rng(n)
    made = [(1010 + 150 * t, random_parents(rng, n)) for t in range(9)]
    assert 9 * n <= 256
    b = _batch(rng, made, [t % shape.r_max for t in range(9)])
    kv, pt = _cache(shape, [(t % shape.r_max, base + n) for t, (base, _) in enumerate(made)], n)
    q = _q(shape, b.n, 9)
    _say(f"[gpu] tree attention {H} x {hd}: 9 trees of {n} together and alone, max_nodes {max_nodes}")
    whole = _attend(shape, kv, b, q, max_nodes)[:b.n]
    for t in range(9):
        idx = np.flatnonzero(b.seq == t)
        sel = torch.from_numpy(idx).cuda()
        got = _attend(shape, kv, b.take(idx), q[sel].contiguous(), max_nodes)[:n]
        assert torch.equal(got, whole[sel]), t
    some = np.arange(0, b.n, 29)
    want, tol = _want(shape, kv, pt, b.take(some), q[torch.from_numpy(some).cuda()])
    _close(whole[torch.from_numpy(some).cuda()], want, tol)


@pytest.mark.parametrize("hd,H", [(64, 4), (128, 2)])
def test_stage_calls_over_several_segments(hd, H):
    """Stage calls over contexts past one segment, whose records stand behind the stage's own scratch: at capacity and of
    exactly the rows the same bits, and every tree alone too."""
    from test_gpu_tree_stages import Verify, _restore, _snapshot
    shape = cdbgen.shrink(cdbgen.TINY, name=f"long-{H}x{hd}", d=H * hd, n_heads=H, head_dim=hd, d_ff=96)
    rng = np.random.default_rng(hd)
    v = Verify(shape, cdbgen.model_weights(shape), [(b, random_parents(rng, n)) for b, n in ((1100, 7), (3, 4), (2300, 9))],
               tree.KV_FULL, 12, capacity=64)
    v.state = cdb.State(shape, 64)
    saved, both = _snapshot(v), []
    _say(f"[gpu] stage calls {H} x {hd} over 1100, 3 and 2300 positions")
    for exact in (True, False):
        _restore(v, saved)
        n = v.n if exact else 64
        c, dep = np.zeros(n), np.full(n, 2)
        if exact:
            rows, see, tok = v.pick(np.arange(v.n), c, dep)
        else:
            rows, see, tok = v.laid.rows(np.arange(64), c, dep), v.laid.tree(v.max_nodes), v.laid.tokens
        logits, ids = torch.zeros((n, shape.vocab), device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")
        tree.cdb_tree_prelude(v.model.model, v.kv.c, v.state.c, rows.c, see.c, tok, v.ws.buf)
        tree.cdb_tree_step(v.model.model, v.kv.c, v.state.c, rows.c, see.c, cdb.StepOut(n).c, v.ws.buf)
        tree.cdb_tree_coda(v.model.model, v.kv.c, v.state.c, rows.c, see.c, logits, ids, v.ws.buf)
        torch.cuda.synchronize()
        assert v.error() == 0
        both.append([x[:v.n] if x.dim() == 2 else x for x in _snapshot(v)] + [logits[:v.n].clone(), ids[:v.n].clone()])
    for k, (a, b) in enumerate(zip(*both)):
        assert torch.equal(a, b), k
    for t in range(3):
        _restore(v, saved)
        live = np.flatnonzero(v.row_tree == t)
        rows, see, tok = v.pick(live, np.zeros(len(live)), np.full(len(live), 2))
        logits, ids = torch.zeros((len(live), shape.vocab), device="cuda"), torch.zeros(len(live), dtype=torch.int32, device="cuda")
        tree.cdb_tree_prelude(v.model.model, v.kv.c, v.state.c, rows.c, see.c, tok, v.ws.buf)
        tree.cdb_tree_step(v.model.model, v.kv.c, v.state.c, rows.c, see.c, cdb.StepOut(len(live)).c, v.ws.buf)
        tree.cdb_tree_coda(v.model.model, v.kv.c, v.state.c, rows.c, see.c, logits, ids, v.ws.buf)
        torch.cuda.synchronize()
        at = torch.from_numpy(live).cuda()
        assert torch.equal(logits, both[0][-2][at]) and torch.equal(ids, both[0][-1][at]), t
