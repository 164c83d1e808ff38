"""Performance cases of the operators over chunks of new tokens, and of the sampled verification of drafted tokens.

The program behind these cases serves a looped language model to many users at once.  One call takes the new tokens of
several sequences, a chunk of one to thousands each (a decoded token, a drafted chain, a prompt or a part of one): it
normalises queries and keys head by head, rotates them to their positions and writes keys and values into the paged,
depth-indexed cache (write), and attends over it (attention).  Users that sample have their drafted trees verified
against the target's and the drafter's probabilities (sample).  Widths are those of the two model families that the
tests and the benchmark use (Ouro 1.4B: 16 x 128 heads, r_max 4; Huginn 3.5B: 55 x 96 heads, r_max 32) and of the tests'
tiny model (4 x 64 heads).

A case is a dict with "op" and, by operator:
  write      chunks chunks of rows_lo..rows_hi tokens behind lo..hi committed positions; type of q, k and v ("bf16",
             "fp32"; the written q has it too), norm: RMSNorm of every query and key head, with gains
  attention  the same, and ones chunks of a single token before them; order of the output ("rows", "fragments")
  sample     trees of up to nodes drafted tokens; drafter "dense" (its logits are given) or "sure" (an n-gram table:
             every guess has probability 1), near: how close the drafter's logits are to the target's
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# heads, head_dim, r_max, vocabulary
MODELS = {"tiny": (4, 64, 4, 1024), "ouro": (16, 128, 4, 49152), "huginn": (55, 96, 32, 65536)}
PAGE = 16
MAX_ROWS = 256  # of drafted trees in one call
LAYERS, LAYER = 2, 1
EPS, BASE = 1e-6, 10000.0


def listed():
    return [
        # eight users decode one token each: the smallest call, where latency counts
        dict(op="write", name="write_8_tokens", model="ouro", chunks=8, rows_lo=1, rows_hi=1, lo=100, hi=900, type="bf16",
             norm=True),
        # parts of a few prompts, of odd lengths, from projections that end in 32 bits, heads of 96
        dict(op="write", name="write_7_ragged_huginn", model="huginn", chunks=7, rows_lo=3, rows_hi=201, lo=0, hi=1500,
             type="fp32", norm=True),
        # whole prompts of a batch, the largest write
        dict(op="write", name="write_16_prompts", model="ouro", chunks=16, rows_lo=384, rows_hi=512, lo=0, hi=0,
             type="bf16", norm=True),
        # a drafted chain of one user, over a short chat: the smallest attention
        dict(op="attention", name="attn_one_chain_13", model="ouro", ones=0, chunks=1, rows_lo=13, rows_hi=13, lo=700,
             hi=700, type="bf16", order="rows"),
        # one prompt chunk of the prefill's size, q kept in 32 bits
        dict(op="attention", name="attn_prompt_512_fp32", model="ouro", ones=0, chunks=1, rows_lo=512, rows_hi=512, lo=512,
             hi=512, type="fp32", order="fragments"),
        # several prompts' odd chunks at different depths of the cache, heads of 96
        dict(op="attention", name="attn_9_ragged_huginn", model="huginn", ones=0, chunks=9, rows_lo=33, rows_hi=333, lo=0,
             hi=2047, type="bf16", order="rows"),
        # a decoding batch with two prompts admitted into it: single tokens over long contexts beside long chunks
        dict(op="attention", name="attn_62_decode_2_prompts", model="ouro", ones=62, chunks=2, rows_lo=700, rows_hi=1000,
             lo=2048, hi=4100, type="bf16", order="rows"),
        # four long prompts, each in its second half: the largest
        dict(op="attention", name="attn_4x2048_long", model="ouro", ones=0, chunks=4, rows_lo=2048, rows_hi=2048, lo=4096,
             hi=4096, type="bf16", order="rows"),
        # one user's drafted tree
        dict(op="sample", name="sample_one_tree_13", model="ouro", trees=1, nodes=13, ragged=False, drafter="dense",
             near=0.5),
        # the whole batch drafts chains of four
        dict(op="sample", name="sample_64x4", model="ouro", trees=64, nodes=4, ragged=False, drafter="dense", near=0.5),
        # few sequences, the widest trees, every one of its own size
        dict(op="sample", name="sample_4x64_huginn", model="huginn", trees=4, nodes=64, ragged=True, drafter="dense",
             near=0.7),
        # guesses from an n-gram table, no drafter's probabilities
        dict(op="sample", name="sample_20x9_sure", model="ouro", trees=20, nodes=9, ragged=True, drafter="sure", near=0.7),
    ]


def draw(rng):
    """Sizes log-uniform over the ranges of the listed cases."""
    def logint(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(("write", "attention", "attention", "attention", "sample", "sample"))
    if op == "sample":
        nodes = logint(1, 64)
        return dict(op=op, model=rng.choice(("tiny", "ouro", "huginn")), trees=logint(1, MAX_ROWS // nodes), nodes=nodes,
                    ragged=rng.random() < 0.6, drafter=rng.choice(("dense", "dense", "sure")),
                    near=round(rng.uniform(0.2, 1.5), 3))
    model = rng.choice(("tiny", "ouro", "ouro", "huginn"))
    d = MODELS[model][0] * MODELS[model][1]
    chunks = logint(1, 64)
    hi = logint(1, 2048 if op == "attention" else 1024)
    hi = max(1, min(hi, 8000 * 2048 // (max(d, 2048) * chunks)))
    case = dict(op=op, model=model, chunks=chunks, rows_lo=max(1, int(hi * rng.uniform(0.2, 1.0))), rows_hi=hi,
                type=rng.choice(("bf16", "bf16", "fp32")))
    if op == "write":
        case["lo"] = rng.choice((0, logint(1, 4000)))
        case["hi"] = case["lo"] + rng.randrange(1 + case["lo"] // 2)
        case["norm"] = rng.random() < 0.7
        return case
    case["ones"] = rng.choice((0, 0, logint(1, 96)))
    # at most the largest listed case's products (half of them where q takes two parts), and its cache
    work = 4 * 2048 * 5120 * 2048 // (2 if case["type"] == "fp32" else 1)
    most = min(work // (d * (chunks * hi + case["ones"])) - hi, 64 * 4100 * 2048 // (d * (chunks + case["ones"])) - hi)
    context = logint(1, max(1, min(8000, most * 2 // 3)))
    case["lo"] = rng.choice((0, context, context))
    case["hi"] = case["lo"] + rng.randrange(1 + case["lo"] // 2)
    case["order"] = rng.choice(("rows", "rows", "fragments"))
    return case


# ------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000 + stream)
    return g


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _dtype(case):
    return torch.bfloat16 if case["type"] == "bf16" else torch.float32


def _sizes(case, seed):
    """Rows and first positions of the chunks: the same numbers of rows at every seed, in another order."""
    lengths = np.random.default_rng([case["chunks"], case["rows_lo"]])
    r = np.random.default_rng([seed, 1])
    n = r.permutation(lengths.integers(case["rows_lo"], case["rows_hi"] + 1, case["chunks"]))
    n = np.concatenate([np.ones(case.get("ones", 0), np.int64), n])
    return n, r.integers(case["lo"], case["hi"] + 1, len(n))


def _prepare_chunks(case, seed):
    """Chunks, their sequences' pages in one core plane each, and the pool."""
    H, hd, R, _ = MODELS[case["model"]]
    n, pos0 = _sizes(case, seed)
    r = np.random.default_rng([seed, 2])
    C, M = len(n), int(n.sum())
    need = (pos0 + n + PAGE - 1) // PAGE
    P = int((case["hi"] + case["rows_hi"] + PAGE - 1) // PAGE)
    # whatever the chunks' own sizes
    pages = (case.get("ones", 0) * ((case["hi"] + PAGE) // PAGE)
             + case["chunks"] * ((case["hi"] + case["rows_hi"] + PAGE - 1) // PAGE))
    ids = r.permutation(pages)[:int(need.sum())].astype(np.int32)
    seq = r.permutation(C).astype(np.int32)
    c = r.integers(0, R, C).astype(np.int32)  # the chunks' loops
    table = np.full((C, R + 2, P), -1, np.int32)
    page = []
    for i, own_ids in enumerate(np.split(ids, np.cumsum(need)[:-1])):
        table[seq[i], c[i] + 1, :need[i]] = own_ids
        page.append(_dev(own_ids, np.int64))
    pool = torch.empty((LAYERS, pages, 2, H, PAGE, hd), dtype=torch.bfloat16, device="cuda")
    pool.normal_(0.0, 1.0, generator=_gen(seed, 3))
    row0 = np.concatenate([[0], np.cumsum(n)])
    return {"case": case, "n": n, "pos0_np": pos0, "rows": M, "page": page, "pool": pool, "table": _dev(table, np.int32),
            "row0": _dev(row0, np.int32), "seq": _dev(seq, np.int32), "pos0": _dev(pos0, np.int32), "c": _dev(c, np.int32),
            "row0_np": row0}


def _prepare_write(case, seed):
    H, hd = MODELS[case["model"]][:2]
    st = _prepare_chunks(case, seed)
    n, pos0, M = st["n"], st["pos0_np"], st["rows"]
    chunk = np.repeat(np.arange(len(n)), n)
    pos = np.arange(M) - st["row0_np"][chunk] + pos0[chunk]
    page = torch.cat([p[_dev(pos[chunk == i] // PAGE, np.int64)] for i, p in enumerate(st["page"])])
    # one projection's output, as it comes: [rows][q, k, v][heads][head_dim]
    qkv = torch.empty((M, 3, H, hd), device="cuda").normal_(0.0, 1.3, generator=_gen(seed, 4)).to(_dtype(case))
    gains = [(1 + 0.2 * torch.randn((hd,), device="cuda", generator=_gen(seed, 5 + k))).to(torch.bfloat16)
             for k in range(2)]
    st.update(pos=_dev(pos, np.int64), page_of=page, qkv=qkv, gains=gains,
              q_out=torch.zeros((M, H * hd), dtype=_dtype(case), device="cuda"))
    return st


def _prepare_attention(case, seed):
    H, hd = MODELS[case["model"]][:2]
    st = _prepare_chunks(case, seed)
    M = st["rows"]
    q = torch.empty((M, H * hd), device="cuda").normal_(0.0, 1.5, generator=_gen(seed, 7)).to(_dtype(case))
    pad = (M + 31) // 32 * 32 if case["order"] == "fragments" else M
    st.update(q=q, out=torch.zeros((pad, H * hd), dtype=torch.bfloat16, device="cuda"))
    return st


def _prepare_sample(case, seed):
    V = MODELS[case["model"]][3]
    r = np.random.default_rng([seed, 8])
    T, N = case["trees"], case["nodes"]
    n, parent = _trees(case, seed)
    rows = int(n.sum())
    row0 = np.cumsum(n) - n
    tree = np.repeat(np.arange(T), n)
    node = np.arange(rows) - row0[tree]
    # logits with a few likely tokens and a long tail; the drafter's are near them
    logits = torch.empty((rows, V), device="cuda").normal_(0.0, 2.5, generator=_gen(seed, 9))
    draft = torch.empty((rows, V), device="cuda").normal_(0.0, case["near"], generator=_gen(seed, 10)).add_(logits)
    up = torch.full((T, N), 1.0, device="cuda")
    temperature = _dev(r.uniform(0.6, 1.1, T), np.float32)
    draft_temperature = _dev(r.uniform(0.7, 1.0, T), np.float32)
    # every node's token comes from the distribution that the drafter had after its parent
    par = parent[tree, node]
    at = _dev(np.where(par < 0, 0, row0[tree] + par), np.int64)
    noise = torch.empty((rows, V), device="cuda").exponential_(1.0, generator=_gen(seed, 11)).log_()
    score = draft[at] / draft_temperature[_dev(tree, np.int64), None] - noise
    picked = score.argmax(-1).int().cpu().numpy()
    tokens = np.zeros((T, N), np.int32)
    tokens[tree, node] = picked
    first = np.where(r.random(T) < 0.95, tokens[:, 0], r.integers(0, V, T)).astype(np.int32)
    seq = r.permutation(T).astype(np.int32)
    st = {"case": case, "n": n, "rows": rows, "row0": _dev(row0, np.int32), "seq": _dev(seq, np.int32),
          "len": _dev(r.integers(16, 4000, T), np.int32), "n_nodes": _dev(n, np.int32), "parent": _dev(parent, np.int32),
          "tokens": _dev(tokens, np.int32), "first": _dev(first, np.int32), "logits": logits,
          "draft": draft if case["drafter"] == "dense" else None, "temperature": temperature,
          "draft_temperature": draft_temperature,
          "u_node": up.uniform_(generator=_gen(seed, 12)).clamp_(max=1 - 2.0 ** -24),
          "u_next": torch.rand((T,), device="cuda", generator=_gen(seed, 13))}
    return st


def _trees(case, seed):
    """Node counts [trees] and parents [trees][nodes]: a root, below it chains that fork now and then."""
    r = np.random.default_rng([seed, 14])
    T, N = case["trees"], case["nodes"]
    n = r.integers((N + 1) // 2, N + 1, T) if case["ragged"] else np.full(T, N)
    back = 1 + (r.exponential(1.0, (T, N)) if N > 4 else np.zeros((T, N))).astype(np.int64)
    parent = np.maximum(np.arange(N)[None, :] - back, 0)
    parent[:, 0] = -1
    parent[np.arange(N)[None, :] >= n[:, None]] = -1
    return n.astype(np.int32), parent.astype(np.int32)


def _handles(st):
    """What a program keeps between calls: descriptors, the workspace, output buffers."""
    import paper_2608_09444_amd as cdb
    from paper_2608_09444_amd import chunk, tree
    case = st["case"]
    H, hd, R, V = MODELS[case["model"]]
    desc = cdb.cdb_model_desc(H * hd, H, hd, 4 * H * hd, V, 0, LAYERS, 0, R, 0, 0, PAGE, EPS, BASE)
    st["desc"] = desc
    if case["op"] == "sample":
        st["ws"] = tree.TreeWorkspace(desc, MAX_ROWS, case["trees"])
        st["drafts"] = tree.Drafts(st["seq"], st["len"], st["n_nodes"], st["parent"], st["tokens"])
        st["sampling"] = tree.Sampling(st["logits"], st["u_node"], st["u_next"], draft_logits=st["draft"],
                                       temperature=st["temperature"], draft_temperature=st["draft_temperature"])
        st["accepted"] = tree.Accepted(case["trees"], case["nodes"])
        return
    C = len(st["n"])
    st["ws"] = chunk.ChunkWorkspace(desc, st["rows"], C)
    st["chunks"] = chunk.Chunks(st["rows"], st["row0"], st["seq"], st["pos0"], st["c"])
    st["kv"] = cdb.cdb_kv(None, st["pool"].data_ptr(), None, 0, st["pool"].shape[1], 0, st["table"].data_ptr(),
                          *st["table"].shape[::2])
    if case["op"] == "write":
        q, k, v = st["qkv"].unbind(1)
        gains = st["gains"] if case["norm"] else (None, None)
        st["in"] = chunk.QKV(q, k, v, norm=case["norm"], q_gain=gains[0], k_gain=gains[1])


def prepare(case, seed):
    st = {"write": _prepare_write, "attention": _prepare_attention, "sample": _prepare_sample}[case["op"]](case, seed)
    if own:
        _handles(st)
    return st


# ------------------------------------------------------------------ plain forms

def _rotated(x, norm, gain, pos, hd):
    """RMSNorm over every head, then the rotation of (j, j + hd / 2) by pos * BASE^(-2j / hd), in 32 bits (angles 64)."""
    x = x.float()
    if norm:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.float()
    j = torch.arange(hd // 2, device="cuda", dtype=torch.float64)
    angle = pos.double()[:, None] * torch.pow(torch.tensor(BASE, dtype=torch.float64, device="cuda"), -2 * j / hd)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_write(st):
    case = st["case"]
    hd = MODELS[case["model"]][1]
    q, k, v = st["qkv"].unbind(1)
    q = _rotated(q, case["norm"], st["gains"][0], st["pos"], hd).flatten(1).to(_dtype(case))
    k = _rotated(k, case["norm"], st["gains"][1], st["pos"], hd).to(torch.bfloat16)
    slot = st["pos"] % PAGE
    st["pool"][LAYER, st["page_of"], 0, :, slot] = k
    st["pool"][LAYER, st["page_of"], 1, :, slot] = v.to(torch.bfloat16)
    return {"q": q, "pool": st["pool"]}


def _fragments(x, pad):
    """Rows [n][d] in the operand order that the output projection reads, padded with zero rows."""
    n, d = x.shape
    full = torch.zeros((pad, d), dtype=x.dtype, device=x.device)
    full[:n] = x
    return full.view(pad // 32, 32, d // 16, 2, 8).permute(0, 2, 3, 1, 4).reshape(pad, d)


def _plain_attention(st):
    H, hd = MODELS[st["case"]["model"]][:2]
    rows = []
    for i, (n, p0) in enumerate(zip(st["n"].tolist(), st["pos0_np"].tolist())):
        at = int(st["row0_np"][i])
        kv = st["pool"][LAYER, st["page"][i]].float().permute(1, 2, 0, 3, 4).reshape(2, H, -1, hd)[:, :, :p0 + n]
        q = st["q"][at:at + n].float().view(n, H, hd).transpose(0, 1) / math.sqrt(hd)
        sc = q @ kv[0].transpose(1, 2).contiguous()
        hide = torch.arange(p0 + n, device="cuda") > torch.arange(p0, p0 + n, device="cuda")[:, None]
        sc = sc.masked_fill(hide, -math.inf)
        e = torch.exp(sc - sc.amax(-1, keepdim=True))
        o = (e @ kv[1].contiguous()) / e.sum(-1, keepdim=True)
        rows.append(o.transpose(0, 1).reshape(n, H * hd))
    out = torch.cat(rows).to(torch.bfloat16)
    return _fragments(out, st["out"].shape[0]) if st["case"]["order"] == "fragments" else out


def _softmax64(x, temperature):
    x = x.double() / temperature.double()[:, None]
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_sample(st):
    """Node by node: a child of the current node is accepted if u q(x) < r(x), with r what is left of the target's
    probabilities after its earlier siblings; if not, r becomes what max(r - q, 0) leaves (a guess of probability 1: r
    without that token).  64 bits throughout, as borders of sums decide."""
    T, N = st["parent"].shape
    V = st["logits"].shape[1]
    dense = st["draft"] is not None
    arange = torch.arange(T, device="cuda")
    cur = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    count = torch.zeros(T, dtype=torch.int64, device="cuda")
    path = torch.full((T, N), -1, dtype=torch.int32, device="cuda")
    left = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    guess = torch.zeros((T, V), dtype=torch.float64, device="cuda")
    row0, n = st["row0"].long(), st["n_nodes"].long()
    last = st["logits"].shape[0] - 1
    for j in range(N):
        x, p = st["tokens"][:, j].long(), st["parent"][:, j].long()
        here = (j < n) & (p == cur)
        root = here & (p < 0)
        child = here & (p >= 0)
        have = left.gather(1, x[:, None])[:, 0]
        said = guess.gather(1, x[:, None])[:, 0] if dense else torch.ones_like(have)
        yes = torch.where(root, x == st["first"], child & (st["u_node"][:, j].double() * said < have))
        no = (child & ~yes)[:, None]
        if dense:
            rest = (left - guess).clamp_(min=0.0)
        else:
            rest = left.scatter(1, x[:, None], 0.0)
        left = torch.where(no, rest / rest.sum(-1, keepdim=True).clamp(min=1e-300), left)
        row = (row0 + j).clamp(max=last)
        left = torch.where(yes[:, None], _softmax64(st["logits"][row], st["temperature"]), left)
        if dense:
            guess = torch.where(yes[:, None], _softmax64(st["draft"][row], st["draft_temperature"]), guess)
        path[arange, count.clamp(max=N - 1)] = torch.where(yes, j, path[arange, count.clamp(max=N - 1)].long()).int()
        cur = torch.where(yes, j, cur)
        count = count + yes
    cdf = left.cumsum(-1)
    nxt = (cdf > (st["u_next"].double() * cdf[:, -1])[:, None]).to(torch.uint8).argmax(-1)
    return {"path": path, "count": count.int(), "next": torch.where(count > 0, nxt.int(), st["first"])}


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"write": _plain_write, "attention": _plain_attention, "sample": _plain_sample}[op](state)
    from paper_2608_09444_amd import chunk, tree
    ws = state["ws"].buf
    if op == "write":
        chunk.cdb_chunk_qkv(state["desc"], state["kv"], state["chunks"].c, 1, LAYER, state["in"].c, state["q_out"], ws)
        return {"q": state["q_out"], "pool": state["pool"]}
    if op == "attention":
        order = chunk.CDB_ORDER_FRAGMENTS if state["case"]["order"] == "fragments" else chunk.CDB_ORDER_ROWS
        chunk.cdb_chunk_attention(state["desc"], state["kv"], state["chunks"].c, 1, LAYER, state["q"], state["out"], ws,
                                  order=order)
        return state["out"]
    tree.cdb_tree_sample(state["desc"], state["drafts"].c, state["row0"], state["first"], state["sampling"].c,
                         state["accepted"].c, ws)
    a = state["accepted"]
    return {"path": a.path, "count": a.count, "next": a.next}


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    H, hd, _, V = MODELS[case["model"]]
    d = H * hd
    if case["op"] == "sample":
        n, parent = _trees(case, 1)
        rows = int(n.sum())
        inner = sum(len(set(parent[t, 1:n[t]].tolist())) for t in range(len(n))) if case["drafter"] == "dense" else 0
        # the target's logits of every row, the drafter's of those with children
        return {"bytes": (rows + inner) * V * 4 + rows * 16 + len(n) * 32, "flops": (rows + inner) * V * 4}
    n, pos0 = _sizes(case, 1)
    M = int(n.sum())
    size = 2 if case["type"] == "bf16" else 4
    if case["op"] == "write":
        return {"bytes": M * d * (3 * size + size + 2 * 2) + M * 4, "flops": M * d * 14}
    pairs = int((n * pos0 + n * (n + 1) // 2).sum())
    return {"bytes": int((n + pos0).sum()) * d * 2 * 2 + M * d * (size + 2), "flops": 4 * pairs * d}


# ------------------------------------------------------------------ 64-bit reference

def exact(case, seed):
    return {"write": _exact_write, "attention": _exact_attention, "sample": lambda *_: None}[case["op"]](case, seed)


def _exact_write(case, seed):
    H, hd = MODELS[case["model"]][:2]
    st = _prepare_write(case, seed)
    pool = st["pool"].double()
    x = st["qkv"].double()
    half = hd // 2
    turn = torch.exp(torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / hd * math.log(BASE)))
    z = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), st["pos"].double()[:, None] * turn)[:, None]

    def turned(y, gain):
        if case["norm"]:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / hd + EPS) * gain.double()
        w = torch.complex(y[..., :half].contiguous(), y[..., half:].contiguous()) * z
        return torch.cat([w.real, w.imag], -1)

    q = turned(x[:, 0], st["gains"][0]).reshape(-1, H * hd)
    slot = st["pos"] % PAGE
    pool[LAYER, st["page_of"], 0, :, slot] = turned(x[:, 1], st["gains"][1])
    pool[LAYER, st["page_of"], 1, :, slot] = x[:, 2]
    return {"q": q, "pool": pool}


def _exact_attention(case, seed):
    H, hd = MODELS[case["model"]][:2]
    st = _prepare_attention(case, seed)
    out = torch.zeros((st["rows"], H, hd), dtype=torch.float64, device="cuda")
    for i in range(len(st["n"])):
        n, p0, at = int(st["n"][i]), int(st["pos0_np"][i]), int(st["row0_np"][i])
        K, V = st["pool"][LAYER, st["page"][i]].double().unbind(1)  # [pages][heads][16][hd]
        for h in range(H):
            k, v = (t[:, h].reshape(-1, hd)[:p0 + n] for t in (K, V))
            sc = torch.mm(st["q"][at:at + n, h * hd:(h + 1) * hd].double(), k.t().contiguous()) / math.sqrt(hd)
            sc.masked_fill_(torch.ones_like(sc, dtype=torch.bool).triu_(p0 + 1), -math.inf)
            out[at:at + n, h] = torch.mm(torch.softmax(sc, -1), v)
    rows = out.view(-1, H * hd)
    return _fragments(rows, st["out"].shape[0]) if case["order"] == "fragments" else rows
