"""GPU: the stage calls over drafted rows against the fp64 oracle, node by node: to the oracle every node is the last
position of a sequence of its own, which holds the context and the node's ancestors.  Both sides start every call from the
same states and K/V entries; bounds are those of the plain stage calls' parity tests (max-abs 2e-2, mean-abs 2e-3 over a
run; K/V entries one bf16 step, 2^-7 relative, or the former).  Then whole rounds of drafting, verification and commit,
eager and captured, against plain decoding."""
import sys

import numpy as np
import pytest
import torch

import cdbgen
import paper_2608_09444_amd as cdb
from lockstep import TOL_MAX, TOL_MEAN
from paper_2608_09444_amd import tree
from test_gpu_tree import ancestors, random_parents

pytestmark = pytest.mark.gpu

PAGE = 16
INJECTED = cdbgen.shrink(cdbgen.TINY, name="tiny-inj-2-2-1", d=192, n_heads=2, head_dim=96, d_ff=320, n_prelude=2,
                         injection=1, exit_kind=1, r_max=3)


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


class Verify:
    """A batch of drafted trees on the device, [(committed positions, parents)], tree t over sequence t, laid out by
    cdb_map_pages and cdb_tree_rows."""

    def __init__(self, shape, weights, trees, layout, seed, capacity=None):
        rng = np.random.default_rng(seed)
        s = self.s = shape
        self.trees, self.R = trees, s.r_max
        T, N = len(trees), max(max(len(p) for _, p in trees), 1)
        self.max_nodes = N
        base = np.array([b for b, _ in trees], np.int32)
        self.n_nodes = np.array([len(p) for _, p in trees], np.int32)
        self.row_tree = np.repeat(np.arange(T), self.n_nodes)
        self.row_node = np.concatenate([np.arange(n) for n in self.n_nodes]).astype(np.int32)
        self.base = base[self.row_tree]
        self.depths_below = np.concatenate([ancestors(p)[1] for _, p in trees]).astype(np.int32)
        self.n = len(self.row_tree)
        self.tokens = rng.integers(0, s.vocab, self.n).astype(np.int32)
        parent, tok = np.full((T, N), -1, np.int32), np.zeros((T, N), np.int32)
        for t, (_, p) in enumerate(trees):
            parent[t, :len(p)] = p
        tok[self.row_tree, self.row_node] = self.tokens
        self.P = int(max((b + n + PAGE - 1) // PAGE for b, n in zip(base, self.n_nodes))) or 1
        pages = T * self.P
        self.model = cdb.DeviceModel(s, weights)
        capacity = capacity or self.n
        self.ws = tree.TreeWorkspace(self.model.desc, capacity, T)
        self.kv = cdb.PagedKV(s, T, self.P, pages, pages * s.r_max, pages)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        for pool in (self.kv.pre, self.kv.core, self.kv.coda):
            pool.normal_(0.0, 1.0, generator=g)
        pools = [tree.PagePool(_dev(rng.permutation(k)), _dev([k])) if L else None
                 for k, L in ((pages, s.n_prelude), (pages * s.r_max, s.n_core), (pages, s.n_coda))]
        tree.cdb_map_pages(self.model.desc, self.kv.page_table, *(p.c if p else None for p in pools), layout,
                           _dev(base + self.n_nodes), _dev(np.zeros(T)), self.ws.buf)
        self.drafts = tree.Drafts(_dev(np.arange(T)), _dev(base), _dev(self.n_nodes), _dev(parent), _dev(tok))
        self.laid = tree.TreeRows(T, capacity)
        tree.cdb_tree_rows(self.drafts.c, self.laid.c, self.ws.buf)
        self.state = cdb.State(s, max(self.n, 1))
        torch.cuda.synchronize()
        assert self.error() == 0 and int(self.laid.n_rows) == self.n
        self.table = self.kv.page_table.cpu().numpy()

    def error(self):
        return cdb.cdb_read_device_error(self.ws.buf)

    def pick(self, live, cs=None, deps=None):
        """The rows of these nodes, slot = node's row, and what they see."""
        at = _dev(live, np.int64)
        rows = cdb.Rows(live, self.laid.seq[at], self.laid.pos[at], cs, deps)
        see = tree.Tree(self.max_nodes, self.laid.base[at], self.laid.mask[at], self.laid.rope_pos[at])
        return rows, see, self.laid.tokens[at]

    def pool(self, plane):
        return self.kv.pre if plane == 0 else self.kv.coda if plane == self.R + 1 else self.kv.core


class AgainstOracle(Verify):
    def __init__(self, shape, weights, trees, layout, seed):
        from oracle_side import OracleSide
        super().__init__(shape, weights, trees, layout, seed)
        # sequence i of the oracle: the context and the ancestors of row i
        self.above = []
        first = np.concatenate([[0], np.cumsum(self.n_nodes)])
        for t, (_, parent) in enumerate(trees):
            for j in range(len(parent)):
                chain, a = [], j
                while a >= 0:
                    chain.append(int(first[t]) + a)
                    a = int(parent[a])
                self.above.append(chain[::-1])
        self.o = OracleSide(shape, weights, [int(b) + len(c) for b, c in zip(self.base, self.above)], kv_layout=layout)
        host = {id(p): p.float().cpu().numpy() for p in (self.kv.pre, self.kv.core, self.kv.coda)}
        for i in range(self.n):
            for plane in self.planes():
                src, dst = host[id(self.pool(plane))], self.o.op.pool_of_plane(plane)
                for pg in range(-(-int(self.base[i]) // PAGE)):
                    dst[self.o.op.page_table[i, plane, pg]] = src[:, self.table[self.row_tree[i], plane, pg]]
        self.sums = {}

    def planes(self):
        s = self.s
        return ([0] if s.n_prelude else []) + list(range(1, self.R + 1)) + ([self.R + 1] if s.n_coda else [])

    def expand(self, live):
        """The oracle's rows for these: themselves, and wherever else they are an ancestor."""
        alive, rows = set(int(i) for i in live), []
        for i in range(self.n):
            rows += [(i, int(self.base[i]) + k, a) for k, a in enumerate(self.above[i]) if a in alive]
        q, pos, node = (np.array(c, np.int32) for c in zip(*rows))
        return q, pos, node

    def own(self, live):
        q = np.asarray(live, np.int32)
        return self.o.slots(q, self.base[q] + self.depths_below[q])

    def close(self, kind, got, want):
        err = np.abs(np.asarray(got, np.float64) - want)
        assert err.max() <= TOL_MAX, (kind, err.max())
        a = self.sums.setdefault(kind, [0.0, 0])
        a[0] += err.sum()
        a[1] += err.size

    def states(self, live, what):
        slots, at = self.own(live), _dev(live, np.int64)
        self.close("h", self.state.h[at].cpu().numpy(), self.o.oh[slots])
        self.state.h[at] = torch.from_numpy(self.o.oh[slots].astype(np.float32)).cuda()
        if self.o.oe is not None:
            self.close("e", self.state.e[at].cpu().numpy(), self.o.oe[slots])
            self.state.e[at] = torch.from_numpy(self.o.oe[slots].astype(np.float32)).cuda()

    def entries(self, i, planes):
        """K/V of row i, compared and then made the oracle's."""
        t, pos = int(self.row_tree[i]), int(self.base[i] + self.row_node[i])
        opos = int(self.base[i] + self.depths_below[i])
        for plane in planes:
            pool, pid = self.pool(plane), int(self.table[t, plane, pos // PAGE])
            got = pool[:, pid, :, :, pos % PAGE].float().cpu().numpy()
            want = self.o.op.pool_of_plane(plane)[self.o.op.page_table[i, plane, opos // PAGE], :, :, :, opos % PAGE]
            err = np.abs(got - want)
            assert (err <= np.maximum(TOL_MAX, np.abs(want) * 2.0 ** -7 * 1.001)).all(), (i, plane, err.max())
            pool[:, pid, :, :, pos % PAGE] = torch.from_numpy(want.astype(np.float32)).cuda().to(torch.bfloat16)

    def prelude(self):
        live = np.arange(self.n)
        q, pos, node = self.expand(live)
        self.o.prelude(q, pos, self.tokens[node])
        rows, see, tok = self.pick(live)
        tree.cdb_tree_prelude(self.model.model, self.kv.c, self.state.c, rows.c, see.c, tok, self.ws.buf)
        torch.cuda.synchronize()
        self.states(live, "prelude")
        for i in live if self.s.n_prelude else ():
            self.entries(i, [0])

    def signal(self, h, before):
        """The exit signal of states h after a loop from `before`."""
        if self.s.exit_kind == 1:
            return np.linalg.norm(h - before, axis=1)
        w = cdbgen.bf16_to_f32(self.w_exit).astype(np.float64)
        z = (h / np.sqrt((h * h).mean(1, keepdims=True) + self.s.rms_eps)) @ w
        return 1 / (1 + np.exp(-z))

    def step(self, live, c, deps):
        live = np.asarray(live)
        q, pos, node = self.expand(live)
        full = np.full(self.n, 0, np.int32)
        full[live] = deps
        self.o.loop(q, pos, np.full(len(q), c, np.int32), full[node])
        rows, see, _ = self.pick(live, np.full(len(live), c), deps)
        out = cdb.StepOut(len(live))
        before = self.state.h[_dev(live, np.int64)].double().cpu().numpy()
        tree.cdb_tree_step(self.model.model, self.kv.c, self.state.c, rows.c, see.c, out.c, self.ws.buf)
        torch.cuda.synchronize()
        gone = np.asarray(deps) == c + 1
        assert out.mask.cpu().numpy().tolist() == gone.astype(int).tolist()
        assert out.counts.tolist() == [int((~gone).sum()), int(gone.sum())]
        assert out.cont[:int((~gone).sum())].tolist() == np.flatnonzero(~gone).tolist()
        assert out.exited[:int(gone.sum())].tolist() == np.flatnonzero(gone).tolist()
        now = self.signal(self.state.h[_dev(live, np.int64)].double().cpu().numpy(), before)
        assert (np.abs(out.score.cpu().numpy() - now) <= 1e-4 + 1e-5 * np.abs(now)).all()
        self.states(live, "step")
        for k, i in enumerate(live):
            self.entries(i, [c + 1] + (list(range(c + 2, self.R + 1)) if gone[k] else []))

    def coda(self):
        live = np.arange(self.n)
        q, pos, node = self.expand(live)
        logits, _ = self.o.coda(q, pos)
        want = logits[[k for k in range(len(q)) if node[k] == q[k]]]
        rows, see, _ = self.pick(live)
        got = torch.zeros((self.n, self.s.vocab), device="cuda")
        ids = torch.zeros(self.n, dtype=torch.int32, device="cuda")
        tree.cdb_tree_coda(self.model.model, self.kv.c, self.state.c, rows.c, see.c, got, ids, self.ws.buf)
        torch.cuda.synchronize()
        self.close("logits", got.cpu().numpy(), want)
        assert torch.equal(ids.long(), got.argmax(1))
        for i in live if self.s.n_coda else ():
            self.entries(i, [self.R + 1])


@pytest.mark.parametrize("shape,layout", [(cdbgen.TINY, tree.KV_FULL), (cdbgen.TINY, tree.KV_FIRST_THEN_SHARED),
                                          (INJECTED, tree.KV_FULL)], ids=["tiny", "tiny-shared", "injected"])
@pytest.mark.parametrize("bases", [(0, 21), (16, 1, 40), (130,)])
def test_stage_calls_are_the_oracles(shape, layout, bases):
    rng = np.random.default_rng(len(bases))
    trees = [(b, random_parents(rng, n)) for b, n in zip(bases, (7, 4, 9))]
    weights = cdbgen.model_weights(shape)
    v = AgainstOracle(shape, weights, trees, layout, 5)
    v.w_exit = weights["w_exit"]
    _say(f"[gpu] {shape.name}: trees over {bases}, {v.n} rows, {sum(len(a) for a in v.above)} rows of the oracle")
    v.prelude()
    deps = rng.integers(1, v.R + 1, v.n).astype(np.int32)
    for c in range(v.R):
        live = rng.permutation(np.flatnonzero(deps > c))  # in any order
        if len(live):
            v.step(live, c, deps[live])
    v.coda()
    assert v.error() == 0
    for kind, (total, n) in v.sums.items():
        _say(f"[gpu]   {kind}: mean error {total / n:.2e}")
        assert total / n <= TOL_MEAN, kind


def _snapshot(v):
    return [t.clone() for t in (v.state.h, v.kv.pre, v.kv.core, v.kv.coda)]


def _restore(v, saved):
    for t, u in zip((v.state.h, v.kv.pre, v.kv.core, v.kv.coda), saved):
        t.copy_(u)


@pytest.mark.parametrize("shape", [cdbgen.TINY, cdbgen.shrink(cdbgen.TINY, name="bare", n_prelude=0, n_coda=0)],
                         ids=["tiny", "bare"])
def test_calls_at_capacity_are_those_of_their_rows(shape):
    """64 rows of capacity, the count in device memory: bit for bit what a call of exactly those rows gives."""
    rng = np.random.default_rng(8)
    for sizes in ([1], [5, 0, 12], [13, 27], [64]):
        v = Verify(shape, cdbgen.model_weights(shape), [(int(rng.integers(0, 90)), random_parents(rng, n)) for n in sizes],
                   tree.KV_FULL, 3, capacity=64)
        _say(f"[gpu] trees of {sizes} in 64 rows of capacity")
        state = cdb.State(shape, 64)
        v.state = state
        for a, junk in zip((v.laid.seq, v.laid.pos, v.laid.base, v.laid.rope_pos, v.laid.tokens, v.laid.mask),
                           (1 << 30, -5, 0x7fffffff, 0x7fffffff, -1, -1)):
            a[v.n:] = junk  # rows past the count do not matter
        saved = _snapshot(v)
        both = []
        for exact in (True, False):
            _restore(v, saved)
            n = v.n if exact else 64
            c, dep = np.zeros(n), np.arange(n) % 2 + 1
            if exact:
                rows, see, tok = v.pick(np.arange(v.n), c, dep)
            else:
                rows, see, tok = v.laid.rows(np.arange(64), c, dep), v.laid.tree(v.max_nodes), v.laid.tokens
            out = cdb.StepOut(n)
            logits, ids = torch.zeros((n, shape.vocab), device="cuda"), torch.full((n,), -7, dtype=torch.int32, device="cuda")
            tree.cdb_tree_prelude(v.model.model, v.kv.c, state.c, rows.c, see.c, tok, v.ws.buf)
            tree.cdb_tree_step(v.model.model, v.kv.c, state.c, rows.c, see.c, out.c, v.ws.buf)
            tree.cdb_tree_coda(v.model.model, v.kv.c, state.c, rows.c, see.c, logits, ids, v.ws.buf)
            torch.cuda.synchronize()
            assert v.error() == 0
            assert ids[v.n:].eq(-7).all()
            both.append(_snapshot(v) + [logits[:v.n].clone(), ids[:v.n].clone(), out.counts.clone(), out.score[:v.n].clone(),
                                        out.exit_next[:v.n].clone()])
        for k, (a, b) in enumerate(zip(*both)):
            assert torch.equal(a, b), k


@pytest.mark.parametrize("lookahead", [False, True])
def test_gated_steps_are_replays_of_their_exits(lookahead):
    """Exits decided by a threshold, then the same loops with those depths given: the same bits."""
    shape = cdbgen.TINY
    rng = np.random.default_rng(2)
    v = Verify(shape, cdbgen.model_weights(shape), [(b, random_parents(rng, n)) for b, n in ((30, 11), (3, 6), (70, 16))],
               tree.KV_FULL, 4)
    live = np.arange(v.n)
    rows, see, tok = v.pick(live)
    tree.cdb_tree_prelude(v.model.model, v.kv.c, v.state.c, rows.c, see.c, tok, v.ws.buf)
    torch.cuda.synchronize()
    saved = _snapshot(v)
    # a threshold between the scores of the first loop
    out = cdb.StepOut(v.n)
    rows, see, _ = v.pick(live, np.zeros(v.n), np.full(v.n, v.R))
    tree.cdb_tree_step(v.model.model, v.kv.c, v.state.c, rows.c, see.c, out.c, v.ws.buf)
    gate = cdb.Gate(float(out.score.median()), lookahead, v.n)
    _restore(v, saved)
    depth, alive = np.full(v.n, v.R), live
    for c in range(v.R):
        rows, see, _ = v.pick(alive, np.full(len(alive), c))
        out = cdb.StepOut(len(alive))
        tree.cdb_tree_step(v.model.model, v.kv.c, v.state.c, rows.c, see.c, out.c, v.ws.buf, gate=gate.c)
        left = out.mask.cpu().numpy() != 0
        depth[alive[left]] = c + 1
        alive = alive[~left]
        if not len(alive):
            break
    torch.cuda.synchronize()
    assert len(set(depth.tolist())) > 1 and v.error() == 0
    want = _snapshot(v)
    _restore(v, saved)
    for c in range(v.R):
        alive = live[depth > c]
        if len(alive):
            rows, see, _ = v.pick(alive, np.full(len(alive), c), depth[alive])
            tree.cdb_tree_step(v.model.model, v.kv.c, v.state.c, rows.c, see.c, cdb.StepOut(len(alive)).c, v.ws.buf)
    torch.cuda.synchronize()
    for k, (a, b) in enumerate(zip(_snapshot(v), want)):
        assert torch.equal(a, b), k


# ------------------------------------------------------------------ whole rounds

class Speculative:
    """Greedy decoding by rounds: pages for the drafts, rows, stage calls, acceptance, commit, and the pages behind the
    accepted positions given back.  A token at position p runs 1 + p % r_max loops."""

    NODES, CAP = 12, 48

    def __init__(self, shape, model, prompts, ends, layout, seed):
        self.s, self.model, self.ends = shape, model, ends
        self.S = S = len(prompts) + 1  # one more that never drafts
        self.T = T = len(prompts)
        self.rng = np.random.default_rng(seed)
        self.P = -(-(max(ends) + self.NODES) // PAGE)
        pages = S * self.P
        self.pages = (pages, pages * shape.r_max, pages)
        self.kv = cdb.PagedKV(shape, S, self.P, *self.pages)
        self.pools = [tree.PagePool.full(n) if L else None
                      for n, L in zip(self.pages, (shape.n_prelude, shape.n_core, shape.n_coda))]
        self.layout = layout
        self.ws = tree.TreeWorkspace(model.desc, 256, S)
        self.mapped = _dev(np.zeros(S))
        self.toks = [list(p) for p in prompts]
        self.length = _dev([len(p) for p in prompts] + [-1])
        self.map(self.length)
        self.seq = _dev(np.arange(T))
        self.first = torch.zeros(T, dtype=torch.int32, device="cuda")
        for q, p in enumerate(prompts):
            cdb.cdb_prefill(model.model, self.kv.c, q, 0, _dev(p), None, self.first[q:], self.ws.buf)
        self.n_nodes, self.parent, self.tok = _dev(np.zeros(T)), _dev(np.zeros((T, self.NODES))), _dev(np.zeros((T, self.NODES)))
        self.drafts = tree.Drafts(self.seq, self.length, self.n_nodes, self.parent, self.tok)
        self.laid = tree.TreeRows(T, self.CAP)
        slots = torch.arange(self.CAP, dtype=torch.int32, device="cuda")
        self.rows, self.see = self.laid.rows(slots), self.laid.tree(self.NODES)
        # each loop's rows, gathered from the ones that the last one left
        self.cols = [self.laid.seq, self.laid.pos, self.laid.base, self.laid.rope_pos, self.laid.mask]
        self.loops, count = [], self.laid.n_rows
        for c in range(shape.r_max):
            slot, depth, out = torch.zeros_like(slots), torch.ones_like(slots), cdb.StepOut(self.CAP)
            seq, pos, base, rope, mask = cols = [torch.zeros_like(x) for x in self.cols]
            rows = cdb.Rows(slot, seq, pos, torch.full_like(slots, c), depth, d_n_rows=count)
            self.loops.append((rows, cols, tree.Tree(self.NODES, base, mask, rope), out))
            count = out.counts[:1]
        self.state = cdb.State(shape, self.CAP)
        self.ids = torch.zeros(self.CAP, dtype=torch.int32, device="cuda")
        self.logits = torch.zeros((self.CAP, shape.vocab), device="cuda")
        self.acc = tree.Accepted(T, self.NODES)
        torch.cuda.synchronize()

    def map(self, need):
        tree.cdb_map_pages(self.model.desc, self.kv.page_table, *(p.c if p else None for p in self.pools), self.layout,
                           need, self.mapped, self.ws.buf)

    def round(self):
        """Everything on the current stream; no step waits for the host."""
        m, buf = self.model.model, self.ws.buf
        self.map(self.length + torch.cat([self.n_nodes, torch.zeros_like(self.n_nodes[:1])]))
        tree.cdb_tree_rows(self.drafts.c, self.laid.c, buf)
        tree.cdb_tree_prelude(m, self.kv.c, self.state.c, self.rows.c, self.see.c, self.laid.tokens, buf)
        at = torch.arange(self.CAP, device="cuda")
        for rows, cols, see, out in self.loops:
            rows.slot.copy_(at)
            for mine, whole in zip(cols, self.cols):
                mine.copy_(whole[at])
            rows.depth.copy_(1 + see.rope_pos % self.s.r_max)
            tree.cdb_tree_step(m, self.kv.c, self.state.c, rows.c, see.c, out.c, buf)
            at = at[out.cont.long()]
        tree.cdb_tree_coda(m, self.kv.c, self.state.c, self.rows.c, self.see.c, self.logits, self.ids, buf)
        tree.cdb_tree_accept(self.drafts.c, self.laid.row0, self.ids, self.first, self.acc.c, buf)
        tree.cdb_tree_commit(self.model.desc, self.kv.c, self.drafts.c, self.acc.c, buf)
        self.length[:self.T] += self.acc.count
        self.first.copy_(self.acc.next)
        self.map(self.length)

    def draft(self, guess):
        """Trees on the host: the token that is known to follow, then a chain of guesses, each beside a wrong one; no
        nodes for a sequence that is done."""
        n, parent, tok = np.zeros(self.T, np.int32), np.full((self.T, self.NODES), -1, np.int32), \
            np.zeros((self.T, self.NODES), np.int32)
        first, length = self.first.tolist(), self.length.tolist()
        for q in range(self.T):
            if length[q] >= self.ends[q]:
                continue
            at, up = 0, 0
            tok[q, 0] = first[q]
            for k in range(int(self.rng.integers(0, 6))):
                right = int(guess[q][min(length[q] + 1 + k, len(guess[q]) - 1)])
                if self.rng.random() < 0.15:
                    right = (right + 1) % self.s.vocab
                parent[q, at + 1:at + 3], tok[q, at + 1:at + 3] = up, ((right + 7) % self.s.vocab, right)
                at, up = at + 2, at + 2
            n[q] = min(at + 1, self.ends[q] - length[q] + 5)
        for mine, a in ((self.n_nodes, n), (self.parent, parent), (self.tok, tok)):
            mine.copy_(torch.from_numpy(a))
        return int(n.sum())

    def decode(self, guess, captured=False):
        rounds, graph = 0, None
        while self.draft(guess):
            if captured and rounds == 1:  # after one eager round, which sets up what first calls set up
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    self.round()
                torch.cuda.current_stream().wait_stream(side)
            graph.replay() if graph else self.round()
            torch.cuda.synchronize()
            assert cdb.cdb_read_device_error(self.ws.buf) == 0, rounds
            path, count = self.acc.path.tolist(), self.acc.count.tolist()
            for q in range(self.T):
                self.toks[q] += [int(self.tok[q, path[q][i]]) for i in range(count[q])]
                assert path[q] == path[q][:count[q]] + [-1] * (self.NODES - count[q])
                assert count[q] >= (int(self.n_nodes[q]) > 0)  # its root is the token that follows
            assert self.length.tolist()[:self.T] == [len(t) for t in self.toks]
            rounds += 1
            assert rounds < 100
        return rounds


def _plain(shape, model, prompts, toks, end):
    """Decoding one token at a time, fed with toks[q] as far as they go and its own greedy tokens from there: the tokens,
    and every position's logits."""
    T, R = len(prompts), shape.r_max
    P = -(-max(end) // PAGE)
    n = T * P
    kv = cdb.PagedKV(shape, T, P, n, n * R, n)
    pools = [tree.PagePool.full(k).c if L else None
             for k, L in zip((n, n * R, n), (shape.n_prelude, shape.n_core, shape.n_coda))]
    ws = tree.TreeWorkspace(model.desc, 256, T)
    tree.cdb_map_pages(model.desc, kv.page_table, *pools, tree.KV_FULL, _dev(end), _dev(np.zeros(T)), ws.buf)
    state = cdb.State(shape, 1)
    out, step = [], cdb.StepOut(1)
    logits, first = torch.zeros((256, shape.vocab), device="cuda"), torch.zeros(256, dtype=torch.int32, device="cuda")
    for q, p in enumerate(prompts):
        cdb.cdb_prefill(model.model, kv.c, q, 0, _dev(p), logits, first, ws.buf)
        mine, said = list(toks[q]), [None] * (len(p) - 1) + [logits[len(p) - 1].cpu().numpy()]
        for t in range(len(p), end[q]):
            if t == len(mine):
                mine.append(int(said[-1].argmax()))
            rows = cdb.Rows([0], [q], [t])
            cdb.cdb_boundary_prelude(model.model, kv.c, state.c, rows.c, _dev([mine[t]]), ws.buf)
            for c in range(1 + t % R):
                rows = cdb.Rows([0], [q], [t], [c], [1 + t % R])
                cdb.cdb_loop_step(model.model, kv.c, state.c, rows.c, step.c, ws.buf)
            cdb.cdb_boundary_coda(model.model, kv.c, state.c, rows.c, logits, first, ws.buf)
            said.append(logits[0].cpu().numpy())
        out.append((mine, said))
    assert cdb.cdb_read_device_error(ws.buf) == 0
    return out


@pytest.mark.parametrize("shape,layout", [(cdbgen.TINY, tree.KV_FULL),
                                          (cdbgen.shrink(cdbgen.TINY, name="bare", n_prelude=0, n_coda=0), tree.KV_FULL),
                                          (cdbgen.shrink(cdbgen.TINY, name="single", r_max=1), tree.KV_SHARED)],
                         ids=["tiny", "bare", "single"])
def test_rounds_give_the_plain_greedy_tokens(shape, layout):
    """Tokens of whole rounds, eager and captured.  Both decodings' logits lie within the parity bound of the oracle's, so
    a token of one is the other's largest logit, or within four bounds of it."""
    model = cdb.DeviceModel(shape, cdbgen.model_weights(shape))
    prompts = [cdbgen.prompt_ids(shape.vocab, 1, n, stream=q)[0] for q, n in enumerate((5, 16, 31))]
    ends = [40, 47, 60]
    guess = [t for t, _ in _plain(shape, model, prompts, prompts, [e + 8 for e in ends])]
    runs = []
    for captured in (False, True):
        d = Speculative(shape, model, prompts, ends, layout, 6)
        rounds = d.decode(guess, captured)
        new = sum(len(t) for t in d.toks) - sum(len(p) for p in prompts)
        _say(f"[gpu] {shape.name}, captured {captured}: {new} tokens in {rounds} rounds of {len(prompts)} sequences")
        assert new > 1.5 * rounds * 2  # more than one a round, so guesses were accepted
        runs.append((d.toks, d.kv.page_table.clone(), d.kv.pre, d.kv.core, d.kv.coda, d.first, d.length))
        assert d.mapped.tolist() == [-(-len(t) // PAGE) for t in d.toks] + [0]
        d.map(_dev([0] * d.S))  # everything goes back
        for pool, n in zip(d.pools, d.pages):
            assert pool is None or (int(pool.free_count) == n and sorted(pool.free_ids.tolist()) == list(range(n)))
        assert d.kv.page_table.eq(-1).all()
    assert runs[0][0] == runs[1][0]
    for k in range(1, 7):
        assert torch.equal(runs[0][k], runs[1][k]), k
    toks = runs[0][0]
    for q, (_, said) in enumerate(_plain(shape, model, prompts, toks, [len(t) for t in toks])):
        for t in range(len(prompts[q]), len(toks[q])):
            assert said[t - 1][toks[q][t]] >= said[t - 1].max() - 4 * TOL_MAX, (q, t)
