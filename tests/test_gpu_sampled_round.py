"""GPU: the serving round that the chunk calls and sampled acceptance are for, over several rounds: pages mapped, the drafted
chains' q, k and v written, their attention, logits, sampled acceptance, the accepted K/V kept, pages given back.  Eager, and
the same rounds as replays of one captured graph.

The model is one layer whose tokens' projections are rows of a table, so that a token's q, k and v do not depend on how many
rows a call has: every round's cache has to equal, bit for bit, the cache that one call over the whole text writes, though
rejected drafts were written in between.  The attention is held to the 64-bit softmax over that cache, within

  2^-8 |want| + A (2^-16 + S 2^-15 + 2^-19 + n 2^-23)

(fp32 queries; A = sum_s p_s |V_s|, S the largest sum_k |q_k K_sk| / sqrt(hd), n the keys seen: bf16 output, q and weights in
two bf16 parts, 32-bit sums).  Accepted nodes and tokens have to be those of the 64-bit walk over the same logits."""
import math
import sys

import numpy as np
import pytest
import torch

import paper_2608_09444_amd as cdb
from paper_2608_09444_amd import chunk, tree
from test_gpu_tree_sample import sample

pytestmark = pytest.mark.gpu

H, HD, V, PAGE, P = 2, 64, 320, 16, 6
D = H * HD
NODES = (5, 2, 1, 4)     # the known token and the drafted ones, by sequence
PROMPTS = (15, 37, 1, 28)
S, N, M = len(NODES), max(NODES), sum(NODES)
DESC = cdb.cdb_model_desc(D, H, HD, D, V, 0, 1, 0, 1, 0, 0, PAGE, 1e-6, 10000.0)


def _dev(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


class Model:
    def __init__(self, seed):
        g = torch.Generator().manual_seed(seed)
        self.qkv = torch.randn((V, 3, H, HD), generator=g).cuda()
        self.gains = [(1 + 0.2 * torch.randn(HD, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
        self.head = (torch.randn((D, V), generator=g) * 0.4).cuda()
        self.bigram = (torch.randn((V, V), generator=g) * 1.5).cuda()  # the drafter's logits


class Cache:
    def __init__(self, pages):
        self.pool = torch.full((1, pages, 2, H, PAGE, HD), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.table = torch.full((S, 3, P), -1, dtype=torch.int32, device="cuda")
        self.mapped = torch.zeros(S, dtype=torch.int32, device="cuda")
        self.free = tree.PagePool.full(pages)
        self.kv = cdb.cdb_kv(None, self.pool.data_ptr(), None, 0, pages, 0, self.table.data_ptr(), S, P)

    def map(self, length, ws):
        tree.cdb_map_pages(DESC, self.table, None, self.free.c, None, tree.KV_FULL, length, self.mapped, ws)

    def context(self, s, n):
        """K and V of the first n positions of sequence s, [2][heads][n][hd]."""
        ids = self.table[s, 1, :(n + PAGE - 1) // PAGE].cpu().long()
        assert (ids >= 0).all()
        return self.pool[0].cpu()[ids].permute(1, 2, 0, 3, 4).reshape(2, H, -1, HD)[:, :, :n]


def layer(model, cache, chunks, tokens, q, out, ws):
    x = model.qkv.index_select(0, tokens)
    qkv = chunk.QKV(*x.unbind(1), norm=True, q_gain=model.gains[0], k_gain=model.gains[1])
    chunk.cdb_chunk_qkv(DESC, cache.kv, chunks.c, 1, 0, qkv.c, q, ws)
    chunk.cdb_chunk_attention(DESC, cache.kv, chunks.c, 1, 0, q, out, ws)
    return qkv


class Server:
    def __init__(self, model, prompts, first, drafter_is_sure):
        self.model, self.sure = model, drafter_is_sure
        self.cache = Cache(40)
        self.len, self.need, self.first = _dev(PROMPTS), _dev(PROMPTS), _dev(first)
        self.n_nodes = _dev(NODES)
        self.row0 = _dev(np.concatenate([[0], np.cumsum(NODES)]))
        zeros = torch.zeros(S, dtype=torch.int32, device="cuda")
        self.tokens = torch.zeros((S, N), dtype=torch.int32, device="cuda")
        self.noise, self.u_node, self.u_next = (torch.zeros(s, device="cuda") for s in ((N, S, V), (S, N), (S,)))
        self.row_tree = _dev(np.repeat(np.arange(S), NODES), np.int64)
        self.row_node = _dev(np.concatenate([np.arange(n) for n in NODES]), np.int64)
        self.chunks = chunk.Chunks(M, self.row0, _dev(np.arange(S)), self.len, zeros)
        self.drafts = tree.Drafts(_dev(np.arange(S)), self.len, self.n_nodes, _dev(np.tile(np.arange(N) - 1, (S, 1))), self.tokens)
        self.logits, self.draft = (torch.zeros((M, V), device="cuda") for _ in range(2))
        self.temp, self.dtemp = _dev([1.0, 0.7, 1.3, 0.9], np.float32), _dev([1.0, 1.1, 0.8, 1.0], np.float32)
        self.sampling = tree.Sampling(self.logits, self.u_node, self.u_next, None if self.sure else self.draft, self.temp,
                                      None if self.sure else self.dtemp)
        self.acc = tree.Accepted(S, N)
        self.q, self.out = torch.zeros((M, D), device="cuda"), torch.zeros((M, D), dtype=torch.bfloat16, device="cuda")
        self.ws = chunk.ChunkWorkspace(DESC, 128, S).buf
        self.tree_ws = tree.TreeWorkspace(DESC, 64, S).buf
        # the prompts, several chunks of one call
        n = sum(PROMPTS)
        self.cache.map(self.len, self.tree_ws)
        c = chunk.Chunks(n, _dev(np.concatenate([[0], np.cumsum(PROMPTS)])), _dev(np.arange(S)), zeros, zeros.clone())
        layer(model, self.cache, c, _dev(np.concatenate(prompts)), torch.zeros((n, D), device="cuda"),
              torch.zeros((n, D), dtype=torch.bfloat16, device="cuda"), self.ws)
        torch.cuda.synchronize()

    def propose(self, r):
        """Drafted chains and random numbers of a round, from the round's own generator."""
        for t, shape in ((self.noise, (N, S, V)), (self.u_node, (S, N)), (self.u_next, (S,))):
            t.copy_(_dev(r.random(shape, np.float32), np.float32))
        gumbel = -torch.log(-torch.log(self.noise.clamp(1e-7, 1 - 1e-7)))
        self.tokens[:, 0] = self.first
        for j in range(1, N):
            z = self.model.bigram[self.tokens[:, j - 1].long()] / self.dtemp[:, None]
            self.tokens[:, j] = (z if self.sure else z + gumbel[j]).argmax(1).int()
        rows = self.tokens[self.row_tree, self.row_node]
        self.row_tokens = rows
        self.draft.copy_(self.model.bigram[rows.long()])

    def round(self):
        """All calls of a round, nothing of which waits for the host."""
        torch.add(self.len, self.n_nodes, out=self.need)
        self.cache.map(self.need, self.tree_ws)
        self.held = layer(self.model, self.cache, self.chunks, self.graph_tokens, self.q, self.out, self.ws)
        torch.mm(self.out.float(), self.model.head, out=self.logits)
        self.logits.add_(self.draft)  # the drafter is somewhat like the model
        tree.cdb_tree_sample(DESC, self.drafts.c, self.row0, self.first, self.sampling.c, self.acc.c, self.tree_ws)
        tree.cdb_tree_commit(DESC, self.cache.kv, self.drafts.c, self.acc.c, self.tree_ws)

    def finish(self):
        self.len.add_(self.acc.count)
        self.first.copy_(self.acc.next)
        self.cache.map(self.len, self.tree_ws)
        torch.cuda.synchronize()


def check_round(sv, texts, length, first):
    """texts: committed tokens by sequence before the round; returns them after it."""
    n = [len(t) for t in texts]
    assert length.tolist() == n
    tokens, out, q = sv.tokens.cpu().numpy(), sv.out.cpu().double(), sv.q.cpu().double().view(M, H, HD)
    path, count, nxt = (x.cpu().numpy() for x in (sv.acc.path, sv.acc.count, sv.acc.next))
    logits, draft, un, ux = (x.cpu().numpy() for x in (sv.logits, sv.draft, sv.u_node, sv.u_next))
    temp, dtemp = sv.temp.cpu().numpy(), sv.dtemp.cpu().numpy()
    fresh = Cache(40)
    ws = chunk.ChunkWorkspace(DESC, 512, S).buf
    tws = tree.TreeWorkspace(DESC, 1, S).buf
    whole = [np.concatenate([t, tokens[s, :NODES[s]]]) for s, t in enumerate(texts)]
    sizes = [len(w) for w in whole]
    fresh.map(_dev(sizes), tws)
    zeros = torch.zeros(S, dtype=torch.int32, device="cuda")
    c = chunk.Chunks(sum(sizes), _dev(np.concatenate([[0], np.cumsum(sizes)])), _dev(np.arange(S)), zeros, zeros.clone())
    layer(sv.model, fresh, c, _dev(np.concatenate(whole)), torch.zeros((sum(sizes), D), device="cuda"),
          torch.zeros((sum(sizes), D), dtype=torch.bfloat16, device="cuda"), ws)
    torch.cuda.synchronize()
    row, after = 0, []
    for s in range(S):
        K, W = fresh.context(s, sizes[s])
        kept = n[s] + int(count[s])
        got = sv.cache.context(s, kept)  # rejected positions may be on pages given back
        assert torch.equal(got.view(torch.int16), torch.stack([K, W])[:, :, :kept].contiguous().view(torch.int16))
        K, W = K.double(), W.double()
        x = q[row:row + NODES[s]].transpose(0, 1)
        hide = torch.arange(sizes[s])[None] > torch.arange(n[s], sizes[s])[:, None]
        p = torch.softmax((x @ K.transpose(1, 2) / math.sqrt(HD)).masked_fill(hide, -math.inf), -1)
        want, A = p @ W, p @ W.abs()
        big = (x.abs() @ K.abs().transpose(1, 2) / math.sqrt(HD)).masked_fill(hide, 0).amax(-1, keepdim=True)
        keys = (~hide).sum(-1)[None, :, None].double()
        tol = want.abs() * 2 ** -8 + A * (2 ** -16 + big * 2 ** -15 + 2 ** -19 + keys * 2 ** -23)
        err = (out[row:row + NODES[s]].view(NODES[s], H, HD).transpose(0, 1) - want).abs()
        assert (err <= tol).all(), (s, float((err / tol).max()))
        a, b, bad = sample(NODES[s], np.arange(N) - 1, tokens[s], first[s], row, logits, None if sv.sure else draft, temp[s],
                           dtemp[s], un[s], ux[s], V)
        assert not bad and b == nxt[s] and a == path[s, :count[s]].tolist() and len(a) == count[s] >= 1
        after.append(np.concatenate([texts[s], tokens[s, :count[s]]]))
        row += NODES[s]
    return after


@pytest.mark.parametrize("sure", [False, True])
def test_rounds_eager_and_captured(sure):
    print(f"rounds sure={sure}", flush=True)
    sys.stdout.flush()
    r = np.random.default_rng(5)
    model = Model(5)
    prompts = [r.integers(0, V, n) for n in PROMPTS]
    first = r.integers(0, V, S)
    eager, replayed = (Server(model, prompts, first, sure) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    texts, counts = prompts, []
    for i in range(8):
        for sv in (eager, replayed):
            sv.propose(np.random.default_rng(100 + i))
        length, known = eager.len.cpu(), eager.first.cpu().numpy()
        eager.graph_tokens = eager.row_tokens
        eager.round()
        if i == 0:  # captured calls do not run: the first replay is round 0
            replayed.graph_tokens = replayed.row_tokens.clone()
            torch.mm(replayed.out.float(), model.head)
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                replayed.round()
        replayed.graph_tokens.copy_(replayed.row_tokens)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager.acc.path, replayed.acc.path) and torch.equal(eager.acc.next, replayed.acc.next)
        assert torch.equal(eager.out, replayed.out) and torch.equal(eager.cache.table, replayed.cache.table)
        texts = check_round(eager, texts, length, known)
        counts.append(eager.acc.count.cpu().numpy())
        for sv in (eager, replayed):
            sv.finish()
        assert torch.equal(eager.len, replayed.len) and torch.equal(eager.cache.free.free_ids, replayed.cache.free.free_ids)
    for sv in (eager, replayed):
        assert cdb.cdb_read_device_error(sv.ws) == 0 and cdb.cdb_read_device_error(sv.tree_ws) == 0
        assert int(sv.cache.free.free_count.cpu()) == 40 - sum((len(t) + PAGE - 1) // PAGE for t in texts)
    counts = np.array(counts)
    assert counts.max() > 1 and (counts < np.array(NODES)).any()  # some drafts were accepted, some were not
