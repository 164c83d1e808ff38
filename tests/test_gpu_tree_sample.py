"""GPU: sampled acceptance of drafted trees against a plain 64-bit implementation on the host, token for token.

Accepted nodes and tokens are whole numbers and have to be equal.  Both sides work in 64 bits, so they could differ only
where a random number lies within about 1e-13 of a border; the inputs are fixed by their seeds and none does."""
import sys

import numpy as np
import pytest
import torch

import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import tree

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _desc(V):
    return cdb.cdb_model_desc(64, 1, 64, 64, V, 0, 1, 0, 1, 0, 0, 16, 1e-6, 10000.0)


def softmax(x, t):
    x = x.astype(np.float64) / np.float64(np.float32(t))
    e = np.exp(x - x.max())
    return e / e.sum()


def sample(n, parent, tokens, first, row0, logits, draft, temp, dtemp, u_node, u_next, V):
    """Path, next token, and whether the walk met logits that are no distribution, of one tree."""
    cur, path, rejected, r, q = -1, [], [], None, None
    for j in range(n):
        if parent[j] != cur or parent[j] >= j:
            continue
        x = tokens[j]
        if cur < 0:
            if x != first:
                continue
            yes = True
        else:
            if not (0 <= x < V):
                continue
            if r is None or (draft is not None and q is None):
                return path, -1, True
            yes = float(u_node[j]) * (q[x] if draft is not None else 1.0) < r[x]
        if yes:
            path.append(j)
            cur = j
            r = distribution(logits[row0 + j], temp)
            q = None if draft is None else distribution(draft[row0 + j], dtemp)
        else:
            if draft is not None:
                rest = np.maximum(r - q, 0)
            else:
                rest = r.copy()
                rest[x] = 0
            if rest.sum() > 0:
                r = rest / rest.sum()
    if not path:
        return path, first, False
    if r is None:
        return path, -1, True
    c = np.cumsum(r)
    hit = np.flatnonzero(c > float(u_next) * c[-1])
    return path, int(hit[0]) if len(hit) else int(np.flatnonzero(r > 0)[-1]), False


def distribution(x, t):
    if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return None
    return softmax(x, t)


class Case:
    """Trees with logits; tokens drawn from the drafter, so that much is accepted and much is not."""

    def __init__(self, V, T, N, seed, dense=True, near=0.5, width=3, spare=0, temps=True, stride=0):
        r = np.random.default_rng(seed)
        self.V, self.T, self.N, self.dense = V, T, N, dense
        self.n = r.integers(max(1, N // 2), N + 1, T).astype(np.int32)
        if T > 3:
            self.n[1] = 0
        self.parent = np.array([[-1] + [max(0, j - 1 - int(r.integers(0, width))) for j in range(1, N)] for _ in range(T)],
                               np.int32).reshape(T, N)
        self.row0 = (np.cumsum(self.n) - self.n).astype(np.int32)
        self.M = int(self.n.sum()) + spare
        self.logits = r.normal(0, 2.5, (self.M, V + stride)).astype(np.float32)
        self.draft = (self.logits + r.normal(0, near, self.logits.shape)).astype(np.float32) if dense else None
        self.temp = r.uniform(0.5, 1.2, T).astype(np.float32) if temps else None
        self.dtemp = r.uniform(0.6, 1.0, T).astype(np.float32) if temps else None
        self.tokens = r.integers(0, V, (T, N)).astype(np.int32)
        for t in range(T):
            for j in range(1, int(self.n[t])):
                row = self.row0[t] + self.parent[t, j]
                x = (self.draft if dense else self.logits)[row, :V]
                self.tokens[t, j] = r.choice(V, p=softmax(x, self.dt(t)))
        self.first = np.where(r.random(T) < 0.9, self.tokens[:, 0], (self.tokens[:, 0] + 1) % V).astype(np.int32)
        self.u_node, self.u_next = r.random((T, N), np.float32), r.random(T, np.float32)
        self.seq, self.length = r.permutation(T).astype(np.int32), np.full(T, 40, np.int32)

    def t(self, t):
        return 1.0 if self.temp is None else self.temp[t]

    def dt(self, t):
        return 1.0 if self.dtemp is None else self.dtemp[t]

    def device(self):
        V = self.V
        self.desc = _desc(V)
        self.d = {k: _dev(getattr(self, k), np.float32) if getattr(self, k) is not None else None
                  for k in ("logits", "draft", "temp", "dtemp", "u_node", "u_next")}
        part = {k: None if self.d[k] is None else self.d[k][:, :V] for k in ("logits", "draft")}
        self.drafts = tree.Drafts(_dev(self.seq), _dev(self.length), _dev(self.n), _dev(self.parent), _dev(self.tokens))
        self.sampling = tree.Sampling(part["logits"], self.d["u_node"], self.d["u_next"], draft_logits=part["draft"],
                                      temperature=self.d["temp"], draft_temperature=self.d["dtemp"])
        self.d_row0, self.d_first = _dev(self.row0), _dev(self.first)
        self.ws = tree.TreeWorkspace(self.desc, 256, self.T)
        self.acc = tree.Accepted(self.T, self.N)
        return self

    def run(self, stream=None):
        tree.cdb_tree_sample(self.desc, self.drafts.c, self.d_row0, self.d_first, self.sampling.c, self.acc.c, self.ws.buf,
                             stream=stream)

    def want(self, refused=()):
        path, count, nxt, bad = np.full((self.T, self.N), -1, np.int32), np.zeros(self.T, np.int32), self.first.copy(), False
        for t in range(self.T):
            if t in refused or self.row0[t] < 0:
                continue
            p, nxt[t], b = sample(int(self.n[t]), self.parent[t], self.tokens[t], self.first[t], int(self.row0[t]),
                                  self.logits[:, :self.V], None if self.draft is None else self.draft[:, :self.V], self.t(t),
                                  self.dt(t), self.u_node[t], self.u_next[t], self.V)
            path[t, :len(p)] = p
            count[t] = len(p)
            bad |= b
        return path, count, nxt, bad

    def check(self, refused=()):
        torch.cuda.synchronize()
        path, count, nxt, bad = self.want(refused)
        assert np.array_equal(self.acc.count.cpu().numpy(), count)
        assert np.array_equal(self.acc.path.cpu().numpy(), path)
        assert np.array_equal(self.acc.next.cpu().numpy(), nxt)
        return count, bad

    def code(self):
        return cdb.cdb_read_device_error(self.ws.buf)


SIZES = [(32, 1, 1), (64, 3, 2), (1024, 16, 16), (4096, 4, 64), (4128, 64, 4), (5000 // 32 * 32, 7, 13), (49152, 5, 9),
         (65536, 2, 30), (131072 + 32, 2, 3)]


@pytest.mark.parametrize("dense", [True, False])
@pytest.mark.parametrize("V,T,N", SIZES)
def test_sampled_acceptance(V, T, N, dense):
    _say(f"sample {V} {T} x {N} dense={dense}")
    for seed in range(3 if V < 10000 else 1):
        c = Case(V, T, N, seed + N, dense, near=(0.5, 1.5, 0.1)[seed]).device()
        c.run()
        _, bad = c.check()
        assert not bad and c.code() == 0


def test_wide_trees_reject_and_accept():
    """All nodes children of one: many rejections in a row, with and without probabilities of the drafter."""
    _say("wide")
    for dense in (True, False):
        for seed in range(4):
            c = Case(256, 4, 64, seed, dense, near=3.0)
            c.parent[:, 1:] = 0
            c.n[:] = 64
            c.row0 = (np.arange(4) * 64).astype(np.int32)
            need = 256
            r = np.random.default_rng(seed)
            c.M = need
            c.logits = r.normal(0, 2.5, (need, 256)).astype(np.float32)
            c.draft = r.normal(0, 2.5, (need, 256)).astype(np.float32) if dense else None
            c.tokens[:, 1:] = r.integers(0, 256, (4, 63))
            c.first = c.tokens[:, 0].copy()
            c.u_node = r.uniform(0.5, 1, (4, 64)).astype(np.float32)
            c.device()
            c.run()
            c.check()


def test_strides_rows_behind_and_no_temperatures():
    _say("strides")
    for dense in (True, False):
        c = Case(1024, 6, 8, 5, dense, spare=7, temps=False, stride=12).device()
        c.run()
        c.check()


def test_masked_logits_and_equal_distributions():
    _say("masked logits")
    c = Case(2048, 12, 10, 7)
    r = np.random.default_rng(7)
    hide = r.random(c.logits.shape) < 0.9
    hide[:, :3] = False
    for t in range(c.T):  # the drafted tokens stay possible for the drafter
        for j in range(1, int(c.n[t])):
            hide[c.row0[t] + c.parent[t, j], c.tokens[t, j]] = False
    c.logits[hide] = -np.inf
    c.draft[np.roll(hide, 1, 1) & hide] = -np.inf
    c.device()
    c.run()
    _, bad = c.check()
    assert not bad and c.code() == 0
    # the drafter is the target: everything on the way is accepted, and nothing would be left by a rejection
    c = Case(512, 8, 12, 8)
    c.draft, c.dtemp = c.logits.copy(), c.temp.copy()
    c.device()
    c.run()
    c.check()
    # all weight on one token: a rejected twin leaves nothing
    for dense in (True, False):
        c = Case(64, 4, 6, 9, dense)
        c.logits[:] = -np.inf
        c.logits[:, 17] = 0
        if dense:
            c.draft[:] = c.logits
        c.tokens[:, 1:] = r.choice([17, 18, 19], (4, 5))
        c.device()
        c.run()
        _, bad = c.check()
        assert not bad and c.code() == 0


@pytest.mark.parametrize("dense", [True, False])
def test_masks_of_the_lowest_value_and_low_temperatures(dense):
    """Tokens masked with the lowest value of fp32 instead of -inf, whole stretches of the vocabulary among them, rows of
    nothing else (the same for every token), temperatures from the smallest one up, and large logits."""
    _say(f"lowest value dense={dense}")
    lowest = np.finfo(np.float32).min
    for seed in range(3):
        c = Case(12320, 8, 7, 40 + seed, dense)
        for x in (c.logits, c.draft) if dense else (c.logits,):
            x[:, 4096:8192] = lowest
            x[:, 12288:] = lowest
        c.logits[-1] = lowest
        c.tokens[:, 1:] = np.where((c.tokens[:, 1:] >= 4096) & (c.tokens[:, 1:] < 8192), 5, c.tokens[:, 1:]) % 12288
        c.device()
        c.run()
        _, bad = c.check()
        assert not bad and c.code() == 0
        c.temp[:] = [2.0 ** -149, 1e-38, 1e-30, 1e-20, 1e-10, 1e-5, 1e-3, 1e30]
        if dense:
            c.dtemp[:] = c.temp[::-1]
        c.device()
        c.run()
        _, bad = c.check()
        assert not bad and c.code() == 0
        c = Case(4128, 8, 7, 50 + seed, dense)
        c.logits *= 1e30
        c.device()
        c.run()
        _, bad = c.check()
        assert not bad and c.code() == 0


def test_sure_drafter_leaves_nothing_of_a_piece():
    """Both possible tokens of the first 4096 are rejected; the smallest random number then falls on the first possible
    token behind them, and so does none of what the differences of their probabilities leave by rounding."""
    _say("nothing of a piece")
    for seed in range(4):
        c = Case(8192, 64, 3, 60 + seed, dense=False)
        r = np.random.default_rng(seed)
        c.n[:] = 3
        c.row0 = (3 * np.arange(64)).astype(np.int32)
        c.parent[:, 1:] = 0
        c.M = 192
        c.logits = r.normal(0, 2, (192, 8192)).astype(np.float32)
        c.logits[:, 0:4200] = -np.inf
        c.tokens[:, 1:] = r.permuted(np.tile(np.arange(4096), (64, 1)), axis=1)[:, :2]
        for t in range(64):
            c.logits[3 * t, c.tokens[t, 1:]] = 5 + r.normal(0, 1, 2)
        c.first = c.tokens[:, 0].copy()
        c.u_node[:] = 1 - 2.0 ** -24
        c.u_next[:] = 0
        c.device()
        c.run()
        count, bad = c.check()
        assert not bad and (count == 1).all() and (c.acc.next.cpu().numpy() == 4200).all()


def test_sure_drafter_with_little_left():
    """Rejected tokens hold all but 1e-2 to 1e-9 of the probabilities."""
    _say("little left")
    for seed in range(6):
        c = Case(8192, 28, 9, 70 + seed, dense=False, temps=False)
        r = np.random.default_rng(seed)
        c.n[:] = 9
        c.row0 = (9 * np.arange(28)).astype(np.int32)
        c.parent[:, 1:] = 0
        c.M = 252
        c.logits = r.normal(0, 1, (252, 8192)).astype(np.float32)
        c.tokens[:, 1:] = r.integers(0, 8192, (28, 8))
        for t in range(28):
            c.logits[9 * t, c.tokens[t, 1:]] = r.uniform(12, 30, 8)
        c.first = c.tokens[:, 0].copy()
        c.u_node = r.uniform(1 - 2.0 ** -seed * 1e-2, 1, (28, 9)).astype(np.float32)
        c.u_node = np.minimum(c.u_node, np.float32(1 - 2.0 ** -24))
        c.device()
        c.run()
        c.check()


def test_random_numbers_at_the_ends():
    _say("ends")
    for u in (0.0, 1 - 2.0 ** -24, 1.0):
        c = Case(1024, 9, 8, 11)
        c.u_next[:] = u
        c.logits[:, -40:] = -np.inf
        c.device()
        c.run()
        c.check()
        c.u_node[:] = min(u, 1 - 2.0 ** -24)
        c.device()
        c.run()
        c.check()


def test_logits_that_are_no_distribution():
    _say("no distribution")
    for value in (np.nan, np.inf, -np.inf):
        for which in ("logits", "draft"):
            c = Case(4128, 6, 8, 13)
            x = getattr(c, which)
            for t in range(6):
                if c.n[t] > 1:
                    row = c.row0[t] + min(1, int(c.n[t]) - 1)
                    if np.isneginf(value):
                        x[row] = value
                    else:
                        x[row, 4100 + t] = value
            c.device()
            c.run()
            _, bad = c.check()
            assert c.code() == (tree.CDB_DEV_BAD_VALUE if bad else 0)
            assert bad
    c = Case(64, 5, 4, 14)
    for k, value in enumerate((0.0, -1.0, np.nan, np.inf)):
        c.temp[k] = value
    c.n[:] = np.minimum(c.n, 2)
    c.device()
    c.run()
    torch.cuda.synchronize()
    assert c.code() == tree.CDB_DEV_BAD_VALUE
    c.check(refused=(0, 1, 2, 3))


def test_refused_trees_and_bad_indices():
    _say("refused")
    c = Case(256, 8, 6, 15)
    c.parent[2, 3] = 5        # never reached
    c.tokens[4, 1] = -1       # not accepted
    c.tokens[5, 1:] = 256
    c.device()
    c.run()
    assert c.code() == cdb.CDB_DEV_BAD_INDEX
    c.check()
    # a repeated sequence, one out of range, a bad length: they stand where the next tree's rows begin
    c = Case(256, 8, 6, 16)
    c.seq[3] = c.seq[2]
    c.seq[5] = 8
    c.length[c.seq[6]] = -1
    gone = (3, 5, 6)
    c.row0 = np.array([sum(int(c.n[k]) for k in range(t) if k not in gone) for t in range(8)], np.int32)
    c.device()
    c.run()
    assert c.code() == cdb.CDB_DEV_BAD_INDEX
    c.check(refused=gone)
    # rows that are not there, trees without rows
    c = Case(256, 5, 6, 17)
    c.row0[2] = -1
    c.device()
    c.run()
    c.check()
    c.n[:] = 0
    c.device()
    c.run()
    c.check()
    assert c.code() == 0


def test_rows_past_the_end():
    """A row0 whose last nodes would lie past the logits: those nodes are not there."""
    _say("rows past the end")
    c = Case(256, 1, 8, 18)
    c.n[:] = 8
    c.parent[:] = np.arange(8) - 1
    c.logits, c.draft = c.logits[:4], c.draft[:4]
    c.M = 4
    c.tokens[0, 0] = c.first[0]
    c.device()
    c.run()
    assert c.code() == cdb.CDB_DEV_BAD_INDEX
    c.n[:] = 4
    c.check()


def test_streams_and_graphs():
    _say("graph")
    c = Case(4128, 12, 10, 19).device()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run()
    for seed in (20, 21, 20):
        o = Case(4128, 12, 10, 19)
        r = np.random.default_rng(seed)
        o.u_node, o.u_next = r.random((12, 10), np.float32), r.random(12, np.float32)
        c.d["u_node"].copy_(_dev(o.u_node, np.float32))
        c.d["u_next"].copy_(_dev(o.u_next, np.float32))
        graph.replay()
        c.u_node, c.u_next = o.u_node, o.u_next
        c.check()
        c.run()
        c.check()


def test_graphs_that_share_a_workspace():
    """Two captured calls, of a dense and of a sure drafter, on one workspace, replayed in turn with an eager one between."""
    _say("two graphs")
    cases = [Case(V, T, N, 23 + N, dense).device() for V, T, N, dense in ((8224, 9, 12, True), (4128, 20, 9, False),
                                                                            (8224, 5, 4, True))]
    for c in cases:
        c.ws = cases[0].ws
    graphs = []
    for c in cases[:2]:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run()
    for _ in range(3):
        for g, c in zip(graphs, cases):
            c.acc.path.fill_(7)
            c.acc.count.fill_(7)
            g.replay()
            c.check()
        cases[2].run()
        cases[2].check()


@pytest.mark.parametrize("dense", [True, False])
def test_largest_vocabulary(dense):
    _say(f"largest vocabulary dense={dense}")
    c = Case(1 << 20, 2, 5, 3, dense, near=1.5).device()
    c.run()
    _, bad = c.check()
    assert not bad and c.code() == 0


def test_tokens_are_distributed_as_the_target():
    """The token that follows a root, accepted or drawn, over 256 trees and 40 seeds against the target's probabilities:
    each of 32 counts of 10240 draws within 5 standard deviations.  The drafter is far off, with three guesses a tree."""
    _say("distribution")
    V, T, N = 32, 64, 4
    r = np.random.default_rng(22)
    for dense in (True, False):
        p_row, q_row = r.normal(0, 1.2, V).astype(np.float32), r.normal(0, 1.2, V).astype(np.float32)
        p, q = softmax(p_row, 1), softmax(q_row, 1)
        got = np.zeros(V)
        c = Case(V, T, N, 23, dense, temps=False)
        c.n[:] = N
        c.row0 = (np.arange(T) * N).astype(np.int32)
        c.M = T * N
        c.parent[:] = [-1, 0, 0, 0]
        c.first = c.tokens[:, 0].copy()
        c.logits = np.tile(p_row, (c.M, 1))
        c.draft = np.tile(q_row, (c.M, 1)) if dense else None
        c.device()
        for _ in range(160):
            tok = r.choice(V, (T, N), p=q).astype(np.int32)
            if not dense:  # distinct guesses
                tok = np.argsort(r.random((T, V)), 1)[:, :N].astype(np.int32)
            tok[:, 0] = c.first
            c.drafts.tokens.copy_(_dev(tok))
            c.d["u_node"].copy_(_dev(r.random((T, N), np.float32), np.float32))
            c.d["u_next"].copy_(_dev(r.random(T, np.float32), np.float32))
            c.run()
            torch.cuda.synchronize()
            count, path, nxt = (x.cpu().numpy() for x in (c.acc.count, c.acc.path, c.acc.next))
            second = np.where(count > 1, tok[np.arange(T), np.maximum(path[:, 1], 0)], nxt)
            got += np.bincount(second, minlength=V)
        n = got.sum()
        assert n == 10240
        assert (np.abs(got - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_roots_outside_the_vocabulary():
    """A root's token outside [0, vocab) is not accepted, and told, also where the token already drawn is the same; a
    good root behind it is taken."""
    _say("roots")
    for dense in (True, False):
        for token in (-1, 256, 2 ** 31 - 1, -2 ** 31):
            c = Case(256, 4, 6, 27, dense)
            c.n[:] = 6
            c.row0 = (6 * np.arange(4)).astype(np.int32)
            c.M = 24
            r = np.random.default_rng(27)
            c.logits = r.normal(0, 2.5, (24, 256)).astype(np.float32)
            c.draft = (c.logits + r.normal(0, 0.5, c.logits.shape)).astype(np.float32) if dense else None
            c.first = c.tokens[:, 0].copy()
            c.tokens[2, 0] = c.first[2] = token
            c.device()
            c.run()
            torch.cuda.synchronize()
            assert c.code() == cdb.CDB_DEV_BAD_INDEX
            got = [x.cpu().numpy() for x in (c.acc.path, c.acc.count, c.acc.next)]
            path, count, nxt, _ = c.want(refused=(2,))
            assert nxt[2] == token and count[2] == 0
            for a, b in zip(got, (path, count, nxt)):
                assert np.array_equal(a, b)
            # a second root
            c.first[2] = 7
            c.parent[2, 1] = -1
            c.tokens[2, 1] = 7
            c.device()
            c.run()
            c.check()
            assert c.code() == cdb.CDB_DEV_BAD_INDEX
