"""Timed cases of decoding with several continuations of a sequence on one paged cache, through the public entry
points: attn_tree, kv_append with parents and kv_keep, verify_tree, beam_select and beam_reorder.

A drafted tree: sequence b owns rows row_start[b] .. row_start[b + 1] - 1 of a chunk, its nodes. Node i sits in the
cache at position ctx_len[b] + i and names an earlier node of the sequence as its parent (-1: none, it follows the
context). A node sees the context, its ancestors and itself, and is rotated by ctx_len[b] + its depth.

    attn     softmax(scale q K^T) V over what each node sees
    step     what a step does with the caches of all layers: rotate q and k and write k and v of the nodes, keep the
             accepted path (position path[b, j] of the nodes moves to position j), read the kept rows back
    verify   a token is drawn from every node's distribution; from the root on, the child that holds the drawn token
             is accepted, until there is none
    select   log softmax(logits) + score, the best K of a group's beams and vocabulary (a finished beam stands for itself)
    reorder  beam b goes on from beam parent[b]: full pages are shared through the table, the last, partly filled page
             is copied into a page of a beam that nobody goes on from; the partly filled pages are read back

Cache layouts are those of the paged cache: keys [pages, kv heads, page, d], values [pages, kv heads, page / 32, d, 32]
with position t of a block of 32 in slot 8 ((t % 16) / 4) + 4 (t / 16) + t % 4, int8 scales fp16 [pages, kv heads, page].
"""
import math

import torch

own = False

VOCAB = 32000
BLK = 32
SLOT = [8 * ((t & 15) >> 2) + 4 * (t >> 4) + (t & 3) for t in range(BLK)]
EOS, PAD = 2, 0


def _named(c, name):
    return c if name is None else dict(c, name=name)


def _attn(name, heads, kv_heads, d, kvq, page, B, ctx, nodes, ragged):
    return _named({"kind": "attn", "heads": heads, "kv_heads": kv_heads, "d": d, "kvq": kvq, "page": page, "B": B,
                   "ctx": ctx, "nodes": nodes, "ragged": ragged}, name)


def _step(name, heads, kv_heads, d, kvq, page, B, ctx, nodes, ragged, layers):
    return dict(_attn(name, heads, kv_heads, d, kvq, page, B, ctx, nodes, ragged), kind="step", layers=layers)


def _verify(name, B, nodes, ragged, vocab, temperature):
    return _named({"kind": "verify", "B": B, "nodes": nodes, "ragged": ragged, "vocab": vocab, "temperature": temperature}, name)


def _select(name, groups, beams, best, vocab, done):
    return _named({"kind": "select", "groups": groups, "beams": beams, "best": best, "vocab": vocab, "done": done}, name)


def _reorder(name, kv_heads, d, kvq, page, groups, beams, ctx, layers):
    return _named({"kind": "reorder", "kv_heads": kv_heads, "d": d, "kvq": kvq, "page": page, "groups": groups,
                   "beams": beams, "ctx": ctx, "layers": layers}, name)


def listed():
    return [
        # one user's small tree over a short context (7B shape): the smallest call, latency
        _attn("tree-one", 32, 32, 128, "bf16", 64, 1, 331, 8, False),
        # a serving batch's trees, contexts of all lengths, grouped queries, int8 cache
        _attn("tree-batch", 64, 8, 128, "int8", 64, 32, 8192, 16, False),
        # the largest trees far into long contexts, 70B tensor-parallel shard
        _attn("tree-long", 8, 1, 128, "bf16", 256, 8, 30001, 64, False),
        # trees of different sizes in one call, odd sizes, head_dim 64
        _attn("tree-odd", 24, 6, 64, "bf16", 96, 17, 1777, 23, True),
        # one sequence's nodes enter the caches of two layers and its accepted path stays
        _step("step-one", 32, 32, 128, "bf16", 64, 1, 331, 8, False, 2),
        # a batch's, four layers of int8 caches, grouped heads, trees of different sizes
        _step("step-batch", 64, 8, 128, "int8", 64, 40, 3000, 27, True, 4),
        # one sequence's tree against greedy decoding
        _verify("verify-one", 1, 8, False, VOCAB, 0.0),
        # a batch's trees of different sizes, sampled
        _verify("verify-batch", 16, 48, True, VOCAB, 0.8),
        # four beams of one request
        _select("select-one", 1, 4, 4, VOCAB, False),
        # a batch of requests with eight beams each over a large vocabulary, twice as many candidates as beams
        _select("select-batch", 24, 8, 16, 128000, True),
        # four beams' caches change places in two layers
        _reorder("reorder-one", 32, 128, "bf16", 64, 1, 4, 331, 2),
        # a batch's, four layers of int8 caches in large pages
        _reorder("reorder-batch", 8, 128, "int8", 256, 16, 8, 4001, 4),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """A case of the same ranges: kv heads 1 to 32 with 1 to 16 query heads each, head_dim 64 or 128, either cache
    format, pages of 32 to 256 positions, 1 to 64 sequences with 0 to 32767 positions of context and trees of 1 to 64
    nodes, 1 to 4 layers; 1 to 64 requests of 1 to 16 beams with up to twice as many candidates; vocabularies of 1000
    to 160000 ids."""
    top_b = max(work(c)["bytes"] for c in listed())
    top_f = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["attn", "attn", "step", "verify", "select", "reorder"])
        vocab, B, ragged = _log(rng, 1000, 160000), _log(rng, 1, 64), rng.random() < 0.5
        nkv, g, d = rng.choice([1, 2, 3, 4, 6, 8, 16, 32]), rng.choice([1, 1, 2, 3, 4, 5, 8, 16]), rng.choice([64, 128])
        kvq, page, ctx, nodes = rng.choice(["bf16", "int8"]), 32 * rng.randint(1, 8), _log(rng, 1, 32768) - 1, _log(rng, 1, 64)
        layers, beams = rng.randint(1, 4), _log(rng, 1, 16)
        if kind == "verify":
            c = _verify(None, B, nodes, ragged, vocab, rng.choice([0.0, 0.5, 0.7, 1.0, 1.3]))
        elif kind == "select":
            c = _select(None, B, beams, rng.randint(beams, 2 * beams), vocab, rng.random() < 0.5)
        elif kind == "reorder":
            c = _reorder(None, nkv, d, kvq, page, B, beams, ctx, layers)
        elif nkv * g > 128:
            continue
        elif kind == "step":
            c = _step(None, nkv * g, nkv, d, kvq, page, B, ctx, nodes, ragged, layers)
        else:
            c = _attn(None, nkv * g, nkv, d, kvq, page, B, ctx, nodes, ragged)
        w = work(c)
        # what the plain form holds at a time: the pools, padded keys and values and the scores, in 32 bits
        if kind in ("attn", "step"):
            held = c["B"] * (ctx + nodes + page) * nkv * d * 4 * c.get("layers", 2)
            if kind == "attn":
                held = max(held, c["B"] * c["heads"] * nodes * (ctx + nodes) * 4)
        elif kind == "reorder":
            held = c["groups"] * beams * (ctx + 2 * page) * nkv * d * 4 * layers
        else:
            held = 0
        if w["bytes"] <= top_b and w["flops"] <= top_f and held <= 6 << 30:
            return c


# ------------------------------------------------------------------ sizes that vary inside a case
def _share(i, n):
    """A spread over (0, 1], one for the last."""
    return 1.0 if i == n - 1 else ((i * 7919 + 5) % 97 + 1) / 98.0


def _contexts(c, n):
    return [int(c["ctx"] * _share(i, n)) for i in range(n)]


def _nodes(c):
    return [max(1, round(c["nodes"] * (_share(b, c["B"]) if c["ragged"] else 1.0))) for b in range(c["B"])]


def _kept(n, b):
    """Nodes of a sequence's accepted path, the root among them."""
    return 1 + (b * 31 + 2) % min(n, 7)


def _survivors(c):
    """Beams of a group that others go on from."""
    return max(1, round(0.6 * c["beams"]))


def _per_position(c):
    """Bytes of a position of one layer's cache."""
    return c["kv_heads"] * (2 * c["d"] * (1 if c["kvq"] == "int8" else 2) + (4 if c["kvq"] == "int8" else 0))


def work(c):
    """Bytes and operations of one pass: every input read once, every output written once."""
    if c["kind"] == "verify":
        rows = sum(_nodes(c))
        return {"bytes": 4.0 * rows * c["vocab"] + 12.0 * rows + 8.0 * rows + 4.0 * c["B"], "flops": 4.0 * rows * c["vocab"]}
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        return {"bytes": 4.0 * rows * c["vocab"] + 5.0 * rows + 13.0 * c["groups"] * c["best"], "flops": 4.0 * rows * c["vocab"]}
    per, nkv, d = _per_position(c), c["kv_heads"], c["d"]
    if c["kind"] == "reorder":
        L, W = c["layers"], c["beams"]
        b = f = 0.0
        for x in _contexts(c, c["groups"]):
            part = x % c["page"]
            # copied once in and out, every beam's part read back, the table's shared columns rewritten
            b += L * part * (2 * (W - _survivors(c)) * per + W * (per + 4 * nkv * d)) + 8.0 * W * (x // c["page"] + 1) + 8.0 * W
            f += 2.0 * L * W * part * nkv * d
        return {"bytes": b + 1.0, "flops": f + 1.0}
    H, n, ctx = c["heads"], _nodes(c), _contexts(c, c["B"])
    if c["kind"] == "step":
        keep = sum(_kept(x, b) for b, x in enumerate(n))
        # the nodes' keys and values in, their cache positions and rotated queries out, the path's positions moved and read
        b = sum(n) * (4 * nkv * d + per + (4 * H * d + 4 * d if c["kvq"] == "bf16" else 0)) + keep * (3 * per + 4 * nkv * d)
        return {"bytes": float(c["layers"] * b), "flops": float(c["layers"] * sum(n) * (6 * nkv * d + 3 * H * d))}
    pairs = sum(m * x + 2 * m - 1 for x, m in zip(ctx, n))       # a tree is at least as deep as a star
    total = sum(m + x for x, m in zip(ctx, n))
    return {"bytes": float(total * per + sum(n) * (4 * H * d + 4)), "flops": 4.0 * d * H * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _quantise(x):
    """x [..., d] -> int8 codes and fp16 scales [...]."""
    s = (x.abs().amax(-1) / 127.0).half()
    q = torch.where(s[..., None] > 0, x / s[..., None].float(), torch.zeros_like(x))
    return q.round().clamp(-127, 127).to(torch.int8), s


def _angles(n, d):
    inv = 1e4 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) * 2.0 / d)
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


def _pool(c, g, layers, n_pages):
    """Pages as earlier steps left them, all layers in one tensor: every position holds some token's key and value."""
    nkv, d, ps = c["kv_heads"], c["d"], c["page"]
    chan = torch.exp(0.4 * torch.randn(nkv, 1, d, generator=g, device="cuda"))
    pool = {}
    for name in ("k", "v"):
        x = torch.randn(layers, n_pages, nkv, ps, d, generator=g, device="cuda") * chan
        if name == "k":
            x /= chan.pow(2).mean().sqrt()
        if c["kvq"] == "int8":
            x, pool[name + "_scales"] = _quantise(x)
        else:
            x = x.bfloat16()
        if name == "v":
            y = torch.empty(layers, n_pages, nkv, ps // BLK, d, BLK, dtype=x.dtype, device="cuda")
            y[..., torch.tensor(SLOT, device="cuda")] = x.view(layers, n_pages, nkv, ps // BLK, BLK, d).transpose(-1, -2)
            x = y
        pool[name] = x
    return pool


def _tables(g, need, ps, spare):
    """A table row of shuffled pages for each of `need` positions, and the pages in all."""
    pages = [-(-n // ps) for n in need]
    n_pages = sum(pages) + spare
    perm = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(need), max(pages)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages


def _starts(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _trees(c, g, n, chain=None):
    """A parent for every node, all sequences' after each other: node 0 is the root, others hang on any earlier node, with
    more on the first ones; chain[b]: nodes that follow each other."""
    R = max(n)
    r = torch.rand(len(n), R, generator=g, device="cuda").cpu()
    out = []
    for b, m in enumerate(n):
        p = [-1] + [min(i - 1, int(i * float(r[b, i]) ** 2)) for i in range(1, m)]
        for x, y in zip(chain[b], chain[b][1:]) if chain else ():
            p[y] = x
        out += p
    return _ints(out)


def prepare(c, seed):
    g = _gen(seed)
    s = {"verify": _prepare_verify, "select": _prepare_select, "reorder": _prepare_reorder}.get(c["kind"], _prepare_tree)(c, g)
    s["c"] = c
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the framework keeps: caches, chunks, workspaces."""
    import paper_2501_13111_amd as fp
    c = s["c"]
    if c["kind"] == "verify":
        s["workspace"] = fp.verify_tree_workspace(s["logits"].shape[0], c["vocab"])
        return
    if c["kind"] == "select":
        s["workspace"] = fp.beam_select_workspace(c["groups"], c["beams"], c["best"], c["vocab"])
        return
    pool = s["pool"]
    s["kvs"] = [fp.PagedKV(**{k: v[i] for k, v in pool.items()}) for i in range(pool["k"].shape[0])]
    if c["kind"] == "reorder":
        s["read"] = fp.Chunk(s["read_start"], s["read_ctx"], s["table_out"], max_new=c["page"])
        return
    s["chunk"] = fp.Chunk(s["row_start"], s["ctx_len"], s["table"], max_new=max(_nodes(c)), max_len=s["max_len"])
    if c["kind"] == "attn":
        s["workspace"] = fp.attn_chunk_workspace(s["kvs"][0], s["chunk"], s["q"].shape[0], c["heads"])
    else:
        s["read"] = fp.Chunk(s["read_start"], s["ctx_len"], s["table"], max_new=7, max_len=s["max_len"])


def _prepare_tree(c, g):
    n, ctx = _nodes(c), _contexts(c, c["B"])
    nkv, d, H, L = c["kv_heads"], c["d"], c["heads"], c.get("layers", 1)
    table, n_pages = _tables(g, [x + m for x, m in zip(ctx, n)], c["page"], 3)
    start = _starts(n)
    N, R = start[-1], max(n)
    keep = [_kept(m, b) for b, m in enumerate(n)]
    chain = None
    if c["kind"] == "step":
        # a path of `keep` nodes in increasing order
        pick = torch.rand(c["B"], R, generator=g, device="cuda").cpu()
        chain = [[0] + sorted((pick[b, 1:m].argsort()[:k - 1] + 1).tolist()) for b, (m, k) in enumerate(zip(n, keep))]
    s = {"table": table, "row_start": _ints(start), "ctx_len": _ints(ctx), "parent": _trees(c, g, n, chain),
         "pool": _pool(c, g, L, n_pages), "max_len": max(x + m for x, m in zip(ctx, n)),
         # node i of sequence b: its row, and whether it is there
         "rows": torch.tensor(start[:-1], device="cuda")[:, None] + torch.arange(R, device="cuda"),
         "live": torch.arange(R, device="cuda") < torch.tensor(n, device="cuda")[:, None]}
    s["rows"].clamp_(max=N - 1)
    if c["kind"] == "attn":
        s["q"] = (1.5 * torch.randn(N, H, d, generator=g, device="cuda")).bfloat16()
        s["out"] = torch.empty(N, H, d, dtype=torch.bfloat16, device="cuda")
        return s
    # the columns of one fused projection's output, of every layer
    qkv = torch.randn(L, N, H + 2 * nkv, d, generator=g, device="cuda").bfloat16()
    s["q"], s["k"], s["v"] = qkv[:, :, :H], qkv[:, :, H:H + nkv], qkv[:, :, H + nkv:]
    s["cos"], s["sin"] = _angles(s["max_len"], d)
    s["q_out"] = torch.empty(L, N, H, d, dtype=torch.bfloat16, device="cuda")
    s["path"] = _ints([x + [-1] * (7 - len(x)) for x in chain])
    s["n_keep"], s["read_start"] = _ints(keep), _ints(_starts(keep))
    s["k_out"] = torch.empty(L, sum(keep), nkv, d, dtype=torch.bfloat16, device="cuda")
    s["v_out"] = torch.empty_like(s["k_out"])
    # of every kept row: its sequence and its place on the path
    s["seq"] = torch.tensor([b for b, k in enumerate(keep) for _ in range(k)], device="cuda")
    s["place"] = torch.tensor([j for k in keep for j in range(k)], device="cuda")
    return s


def _logits(g, rows, vocab):
    """Logits with a few likely tokens per row."""
    z = 2.5 * torch.randn(rows, vocab, generator=g, device="cuda")
    return z.scatter_add_(1, torch.randint(vocab, (rows, 8), generator=g, device="cuda"), 9 * torch.rand(rows, 8, generator=g, device="cuda"))


def _prepare_verify(c, g):
    n = _nodes(c)
    start, R = _starts(n), max(n)
    N, V = start[-1], c["vocab"]
    z = _logits(g, N, V)
    parent = _trees(c, g, n)
    first = torch.repeat_interleave(torch.tensor(start[:-1], device="cuda"), torch.tensor(n, device="cuda"))
    # a child holds one of its parent's likely tokens
    T = c["temperature"]
    up = (first + parent.long().clamp(min=0))
    noisy = z[up] / max(T, 0.25) - torch.log(-torch.log(torch.rand(N, V, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    s = {"logits": z, "row_start": _ints(start), "parent": parent, "ids": noisy.argmax(-1).int(),
         "u": torch.rand(N, generator=g, device="cuda"),
         "out_ids": torch.empty(c["B"], R, dtype=torch.int32, device="cuda"),
         "path": torch.empty(c["B"], R, dtype=torch.int32, device="cuda"),
         "n_out": torch.empty(c["B"], dtype=torch.int32, device="cuda"),
         "rows": torch.tensor(start[:-1], device="cuda")[:, None] + torch.arange(R, device="cuda"),
         "live": torch.arange(R, device="cuda") < torch.tensor(n, device="cuda")[:, None]}
    s["rows"].clamp_(max=N - 1)
    return s


def _prepare_select(c, g):
    G, W, K, V = c["groups"], c["beams"], c["best"], c["vocab"]
    # beams agree on much: their logits are a common part and their own
    z = (_logits(g, G, V)[:, None] + 0.7 * torch.randn(G, W, V, generator=g, device="cuda")).view(G * W, V)
    scores = -(12.0 + 4.0 * torch.rand(G, W, generator=g, device="cuda")).sort(-1)[0]
    done = torch.rand(G, W, generator=g, device="cuda") < 0.2 if c["done"] else None
    return {"logits": z, "scores": scores, "done": done,
            "out_scores": torch.empty(G, K, device="cuda"), "out_parent": torch.empty(G, K, dtype=torch.int32, device="cuda"),
            "out_ids": torch.empty(G, K, dtype=torch.int32, device="cuda"),
            "out_done": torch.empty(G, K, dtype=torch.bool, device="cuda")}


def _prepare_reorder(c, g):
    G, W, ps = c["groups"], c["beams"], c["page"]
    ctx = _contexts(c, G)
    table, n_pages = _tables(g, [x + ps for x in ctx for _ in range(W)], ps, 3)
    part, A = [x % ps for x in ctx], _survivors(c)
    # A beams that others go on from, each at least once, in any order
    order = torch.rand(G, W, generator=g, device="cuda").argsort(-1)[:, :A]
    more = order.gather(1, torch.randint(A, (G, W - A), generator=g, device="cuda"))
    parent = torch.cat([order, more], -1)
    parent = parent.gather(1, torch.rand(G, W, generator=g, device="cuda").argsort(-1)).int().contiguous()
    s = {"table": table, "table_out": torch.empty_like(table), "ctx_len": _ints([x for x in ctx for _ in range(W)]), "parent": parent,
         "pool": _pool(c, g, c["layers"], n_pages),
         "read_start": _ints(_starts([x for x in part for _ in range(W)])),
         "read_ctx": _ints([x - p for x, p in zip(ctx, part) for _ in range(W)]),
         "seq": torch.tensor([b for b in range(G * W) for _ in range(part[b // W])], device="cuda", dtype=torch.long),
         "place": torch.tensor([j for b in range(G * W) for j in range(part[b // W])], device="cuda", dtype=torch.long)}
    s["k_out"] = torch.empty(c["layers"], W * sum(part), c["kv_heads"], c["d"], dtype=torch.bfloat16, device="cuda")
    s["v_out"] = torch.empty_like(s["k_out"])
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    kind = s["c"]["kind"]
    if own:
        return _own(s)
    return {"attn": _plain_attn, "step": _plain_step, "verify": _plain_verify, "select": _plain_select,
            "reorder": _plain_reorder}[kind](s)


def _own(s):
    import paper_2501_13111_amd as fp
    c = s["c"]
    if c["kind"] == "attn":
        fp.attn_tree(s["kvs"][0], s["chunk"], s["parent"], s["q"], s["out"], workspace=s["workspace"])
        return s["out"]
    if c["kind"] == "verify":
        fp.verify_tree(s["logits"], s["row_start"], s["parent"], s["ids"], s["u"], s["out_ids"], s["path"], s["n_out"],
                       temperature=c["temperature"], workspace=s["workspace"])
        return s["out_ids"], s["path"], s["n_out"]
    if c["kind"] == "select":
        fp.beam_select(s["logits"], s["scores"], s["out_scores"], s["out_parent"], s["out_ids"], done=s["done"],
                       out_done=s["out_done"], eos_id=EOS, pad_id=PAD, workspace=s["workspace"])
        return s["out_scores"], s["out_parent"], s["out_ids"], s["out_done"]
    out = []
    if c["kind"] == "reorder":
        fp.beam_reorder(s["kvs"], s["table"], s["ctx_len"], s["parent"], table_out=s["table_out"])
        out = [s["table_out"]]
    else:
        for i, kv in enumerate(s["kvs"]):
            if c["kvq"] == "bf16":
                fp.kv_append(kv, s["chunk"], s["k"][i], s["v"][i], q=s["q"][i], q_out=s["q_out"][i], cos=s["cos"],
                             sin=s["sin"], parent=s["parent"])
            else:
                fp.kv_append(kv, s["chunk"], s["k"][i], s["v"][i], parent=s["parent"])
        fp.kv_keep(s["kvs"], s["chunk"], s["path"], s["n_keep"])
        if c["kvq"] == "bf16":
            out = [s["q_out"]]
    for i, kv in enumerate(s["kvs"]):
        fp.kv_read(kv, s["read"], s["k_out"][i], s["v_out"][i])
    return out + [s["k_out"], s["v_out"]]


def _ancestors(s):
    """[sequences, nodes, nodes]: whether node i is node j, or one that j hangs on."""
    R = s["rows"].shape[1]
    p = s["parent"].long()[s["rows"]]
    i = torch.arange(R, device="cuda")
    up = (p[:, None, :] == i[:, None]) & (p >= 0)[:, None, :] & s["live"][:, None, :]
    a = (up | torch.eye(R, dtype=torch.bool, device="cuda")).float()
    for _ in range(6):                       # paths of twice the length each time
        a = (torch.bmm(a, a) > 0).float()
    return a > 0


def _plain_attn(s):
    """All sequences at once, keys and values padded to the longest."""
    c, pool = s["c"], s["pool"]
    ps, nkv, d, H, B = c["page"], c["kv_heads"], c["d"], c["heads"], c["B"]
    G, R, n = H // nkv, s["rows"].shape[1], s["max_len"]
    pages = s["table"][:, :-(-n // ps)].long().clamp(min=0)
    k = pool["k"][0][pages].float()                                        # [B, pages, kv heads, page, d]
    v = pool["v"][0][pages][..., torch.tensor(SLOT, device="cuda")].float().transpose(-1, -2).reshape(B, -1, nkv, ps, d)
    if c["kvq"] == "int8":
        k = k * pool["k_scales"][0][pages].float()[..., None]
        v = v * pool["v_scales"][0][pages].float()[..., None]
    k = k.permute(0, 2, 4, 1, 3).reshape(B * nkv, d, -1)[..., :n].contiguous()
    v = v.permute(0, 2, 1, 3, 4).reshape(B * nkv, -1, d)[:, :n].contiguous()
    ctx, pos = s["ctx_len"].long(), torch.arange(n, device="cuda")
    node = (pos - ctx[:, None]).clamp(0, R - 1)                            # of position p, from ctx on
    tree = _ancestors(s).transpose(1, 2).gather(2, node[:, None, :].expand(B, R, n))
    past = pos >= ctx[:, None] + R
    seen = (pos < ctx[:, None])[:, None, :] | (tree & ~past[:, None, :])   # [B, nodes, positions]
    q = s["q"][s["rows"]].float().view(B, R, nkv, G, d).permute(0, 2, 1, 3, 4).reshape(B * nkv, R * G, d).contiguous()
    sc = torch.bmm(q, k).view(B, nkv, R, G, n) * (1.0 / math.sqrt(d))
    sc.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    e = torch.exp(sc - sc.amax(-1, keepdim=True)).view(B * nkv, R * G, n)
    o = torch.bmm(e, v) / e.sum(-1, keepdim=True)
    o = o.view(B, nkv, R, G, d).permute(0, 2, 1, 3, 4).reshape(B, R, H, d)
    s["out"].copy_(o[s["live"]].bfloat16())
    return s["out"]


def _cached(c, pool, page, off):
    """What the cache holds at (page, offset), of all layers: fp32 [layers, positions, kv heads, d]."""
    slot = torch.tensor(SLOT, device="cuda")[off % BLK]
    k, v = pool["k"][:, page, :, off], pool["v"][:, page, :, off // BLK, :, slot]
    k, v = k.transpose(0, 1).float(), v.transpose(0, 1).float()
    if c["kvq"] == "int8":
        k = k * pool["k_scales"][:, page, :, off].transpose(0, 1).float()[..., None]
        v = v * pool["v_scales"][:, page, :, off].transpose(0, 1).float()[..., None]
    return k, v


def _place(s, seq, pos):
    ps = s["c"]["page"]
    return s["table"][seq, pos // ps].long(), pos % ps


def _move(c, pool, at, to):
    """Positions' contents from (page, offset) `at` to `to`, in all layers: all read before any is written."""
    (pa, oa), (pt, ot) = at, to
    slot = torch.tensor(SLOT, device="cuda")
    k, v = pool["k"][:, pa, :, oa], pool["v"][:, pa, :, oa // BLK, :, slot[oa % BLK]]
    sc = [pool[n][:, pa, :, oa] for n in ("k_scales", "v_scales") if n in pool]
    pool["k"][:, pt, :, ot] = k
    pool["v"][:, pt, :, ot // BLK, :, slot[ot % BLK]] = v
    if sc:
        pool["k_scales"][:, pt, :, ot], pool["v_scales"][:, pt, :, ot] = sc


def _plain_step(s):
    c, pool, d = s["c"], s["pool"], s["c"]["d"]
    seq = torch.arange(c["B"], device="cuda")[:, None].expand_as(s["rows"])[s["live"]]
    node = torch.arange(s["rows"].shape[1], device="cuda").expand_as(s["rows"])[s["live"]]
    depth = _ancestors(s).sum(1)[s["live"]] - 1
    ctx = s["ctx_len"].long()
    page, off = _place(s, seq, ctx[seq] + node)
    slot = torch.tensor(SLOT, device="cuda")[off % BLK]
    k, v = s["k"].float(), s["v"].float()
    out = []
    if c["kvq"] == "bf16":
        cos, sin = s["cos"][ctx[seq] + depth][:, None, :], s["sin"][ctx[seq] + depth][:, None, :]

        def rotate(x):
            lo, hi = x[..., :d // 2], x[..., d // 2:]
            return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

        out = [s["q_out"].copy_(rotate(s["q"].float()).bfloat16())]
        k, v = rotate(k).bfloat16(), v.bfloat16()
    else:
        (k, ks), (v, vs) = _quantise(k), _quantise(v)
        pool["k_scales"][:, page, :, off] = ks.transpose(0, 1)
        pool["v_scales"][:, page, :, off] = vs.transpose(0, 1)
    pool["k"][:, page, :, off] = k.transpose(0, 1)
    pool["v"][:, page, :, off // BLK, :, slot] = v.transpose(0, 1)
    seq, place = s["seq"], s["place"]
    to = _place(s, seq, ctx[seq] + place)
    _move(c, pool, _place(s, seq, ctx[seq] + s["path"].long()[seq, place]), to)
    k, v = _cached(c, pool, *to)
    return out + [s["k_out"].copy_(k.bfloat16()), s["v_out"].copy_(v.bfloat16())]


def _plain_verify(s):
    """Every node's draw in 64 bits (the borders of the draws decide), then the path."""
    c, z, T = s["c"], s["logits"], s["c"]["temperature"]
    if T == 0:
        y = z.argmax(-1)
    else:
        x = z.double() / T
        cum = torch.exp(x - x.amax(-1, keepdim=True)).cumsum(-1)
        y = (cum <= s["u"].double()[:, None] * cum[:, -1:]).sum(-1).clamp(max=c["vocab"] - 1)
    rows, live = s["rows"], s["live"]
    R = rows.shape[1]
    i = torch.arange(R, device="cuda")
    y, p, ids = y[rows], s["parent"].long()[rows], s["ids"].long()[rows]
    hit = (p[:, None, :] == i[:, None]) & (ids[:, None, :] == y[:, :, None]) & live[:, None, :]       # [B, node, child]
    chosen = (hit & (hit.cumsum(-1) == 1)).any(1)                            # of a node's children the first that holds its token
    chosen[:, 0] = True
    on = ((_ancestors(s) & ~chosen[:, :, None]).sum(1) == 0) & live           # all the way down from the root
    # a parent comes before its children: the path in order
    count = on.sum(-1)
    path = torch.where(on, i, i + R).sort(-1)[0]
    last = y.gather(1, path.gather(1, (count - 1)[:, None]))
    inside = i < count[:, None]
    at = path.clamp(max=R - 1)
    nxt = ids.gather(1, torch.cat([at[:, 1:], at[:, :1]], -1))
    s["out_ids"].copy_(torch.where(i + 1 < count[:, None], nxt, torch.where(inside, last, torch.full_like(nxt, -1))))
    s["path"].copy_(torch.where(inside, path, torch.full_like(path, -1)))
    s["n_out"].copy_(count)
    return s["out_ids"], s["path"], s["n_out"]


def _plain_select(s):
    """Scores in 64 bits: the borders decide."""
    c = s["c"]
    G, W, K, V = c["groups"], c["beams"], c["best"], c["vocab"]
    z = s["logits"].double().view(G, W, V)
    m = z.amax(-1, keepdim=True)
    x = s["scores"].double()[..., None] - (m + torch.exp(z - m).sum(-1, keepdim=True).log()) + z
    if s["done"] is not None:
        only = torch.arange(V, device="cuda") == PAD
        x = torch.where(s["done"][..., None], torch.where(only, s["scores"].double()[..., None], float("-inf")), x)
    x = x.view(G, W * V)
    v, at = x.topk(min(2 * K, W * V), -1)
    at, o = at.sort(-1)                                                      # of equal scores the lowest index
    v, o = v.gather(1, o).sort(dim=-1, descending=True, stable=True)
    v, at = v[:, :K], at.gather(1, o)[:, :K]
    none = v == float("-inf")
    parent, ids = torch.where(none, -1, at // V), torch.where(none, -1, at % V)
    was = s["done"].gather(1, parent.clamp(min=0)) if s["done"] is not None else torch.zeros_like(none)
    s["out_scores"].copy_(v)
    s["out_parent"].copy_(parent)
    s["out_ids"].copy_(ids)
    s["out_done"].copy_((was | (ids == EOS)) & ~none)
    return s["out_scores"], s["out_parent"], s["out_ids"], s["out_done"]


def _plain_reorder(s):
    c, pool = s["c"], s["pool"]
    G, W, ps = c["groups"], c["beams"], c["page"]
    p = s["parent"].long()
    beam = torch.arange(W, device="cuda")
    same = p[:, :, None] == p[:, None, :]
    first = (same & (beam[None, :] < beam[:, None])).sum(-1) == 0            # the first of its parent's beams
    taken = (p[:, :, None] == beam).any(1)
    # the k-th of the others takes the partly filled page of the k-th beam that nobody goes on from
    free = torch.where(taken, beam + W, beam).sort(-1)[0] % W
    giver = torch.where(first, p, free.gather(1, ((~first).cumsum(-1) - 1).clamp(min=0)))
    t = s["table"].view(G, W, -1)
    width = t.shape[-1]
    ctx = s["ctx_len"].view(G, W)[:, 0].long()
    full, col = (ctx // ps)[:, None, None], torch.arange(width, device="cuda")
    up, give = t.gather(1, p[..., None].expand_as(t)), t.gather(1, giver[..., None].expand_as(t))
    new = torch.where(col < full, up, torch.where((col == full) & (ctx % ps > 0)[:, None, None], give, t))
    s["table_out"].copy_(new.view(G * W, width))
    # every beam's part from its parent's page; the first of them have it there already
    seq, off = s["seq"], s["place"]
    at = (full[:, 0, 0])[seq // W]
    src, dst = t.reshape(G * W, width)[(seq // W) * W + p.view(-1)[seq], at].long(), s["table_out"][seq, at].long()
    _move(c, pool, (src, off), (dst, off))
    k, v = _cached(c, pool, dst, off)
    return s["table_out"], s["k_out"].copy_(k.bfloat16()), s["v_out"].copy_(v.bfloat16())


# ------------------------------------------------------------------ 64 bits, from the definitions
def exact(c, seed):
    s = prepare(c, seed)
    return {"attn": _exact_attn, "step": _exact_step, "verify": _exact_verify, "select": _exact_select,
            "reorder": _exact_reorder}[c["kind"]](s)


def _read64(s, i, b, p):
    """Key and value at positions p of table row b in layer i, as the cache holds them."""
    c, pool = s["c"], s["pool"]
    pg, off = s["table"][b].long()[p // c["page"]], p % c["page"]
    slot = torch.tensor(SLOT, device="cuda")[off % BLK]
    k, v = pool["k"][i][pg, :, off].double(), pool["v"][i][pg, :, off // BLK, :, slot].double()
    if c["kvq"] == "int8":
        k = k * pool["k_scales"][i][pg, :, off].double()[..., None]
        v = v * pool["v_scales"][i][pg, :, off].double()[..., None]
    return k, v


def _lines(s, b):
    """Of each node of sequence b the nodes from the root down to it."""
    r0, r1 = s["row_start"][b].item(), s["row_start"][b + 1].item()
    out = []
    for i, p in enumerate(s["parent"][r0:r1].tolist()):
        out.append((out[p] if p >= 0 else []) + [i])
    return r0, out


def _exact_attn(s):
    c = s["c"]
    G, d = c["heads"] // c["kv_heads"], c["d"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        ctx = s["ctx_len"][b].item()
        r0, lines = _lines(s, b)
        m = len(lines)
        k, v = _read64(s, 0, b, torch.arange(ctx + m, device="cuda"))
        seen = torch.zeros(m, ctx + m, dtype=torch.bool)
        seen[:, :ctx] = True
        for i, line in enumerate(lines):
            seen[i, [ctx + j for j in line]] = True
        seen = seen.cuda()
        q = s["q"][r0:r0 + m].double()
        for h in range(c["heads"]):
            sc = (q[:, h] @ k[:, h // G].t().contiguous()) / math.sqrt(d)
            out[r0:r0 + m, h] = torch.softmax(sc.masked_fill(~seen, float("-inf")), -1) @ v[:, h // G].contiguous()
    return out


def _exact_step(s):
    c = s["c"]
    d = c["d"]
    depth, take = [], []
    for b in range(c["B"]):
        r0, lines = _lines(s, b)
        depth += [s["ctx_len"][b].item() + len(x) - 1 for x in lines]
        take += [r0 + j for j in s["path"][b].tolist() if j >= 0]
    k, v = s["k"].double(), s["v"].double()
    if c["kvq"] == "int8":
        def held(x):
            # the scale is an fp16 number by definition, the codes are whole numbers
            sc = (x.abs().amax(-1) / 127.0).half().double()[..., None]
            return torch.where(sc > 0, (x / sc).round().clamp(-127, 127) * sc, torch.zeros_like(x))
        return [held(k)[:, take], held(v)[:, take]]
    at = torch.tensor(depth, device="cuda")
    turn = torch.complex(s["cos"].double()[at], s["sin"].double()[at])[:, None, :]

    def rot(x):
        z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
        return torch.cat([z.real, z.imag], -1)
    return [rot(s["q"].double()), rot(k)[:, take], v[:, take]]


def _exact_verify(s):
    """One sequence and one node after another."""
    c, T = s["c"], s["c"]["temperature"]
    parent, ids, u = s["parent"].tolist(), s["ids"].tolist(), s["u"].tolist()
    out, path = torch.full(s["out_ids"].shape, -1, dtype=torch.int32), torch.full(s["path"].shape, -1, dtype=torch.int32)
    count = torch.zeros(c["B"], dtype=torch.int32)
    start = s["row_start"].tolist()
    for b in range(c["B"]):
        r0, m, i = start[b], start[b + 1] - start[b], 0
        while True:
            x = s["logits"][r0 + i].double()
            if T == 0:
                y = int((x == x.max()).nonzero()[0])
            else:
                cum = torch.softmax(x / T, -1).cumsum(-1)
                above = (cum > u[r0 + i] * cum[-1]).nonzero()
                y = int(above[0])
            n = int(count[b])
            out[b, n], path[b, n] = y, i
            count[b] = n + 1
            i = next((j for j in range(m) if parent[r0 + j] == i and ids[r0 + j] == y), None)
            if i is None:
                break
    return out.cuda(), path.cuda(), count.cuda()


def _exact_select(s):
    c = s["c"]
    G, W, K, V = c["groups"], c["beams"], c["best"], c["vocab"]
    lists = [[], [], [], []]
    for g in range(G):
        rows = []
        for w in range(W):
            if s["done"] is not None and bool(s["done"][g, w]):
                rows.append((torch.tensor([PAD], device="cuda"), s["scores"][g, w].double()[None]))
                continue
            x = torch.log_softmax(s["logits"][g * W + w].double(), -1) + s["scores"][g, w].double()
            rows.append((torch.arange(V, device="cuda"), x))
        best = []
        for w, (ids, x) in enumerate(rows):
            top = x.topk(min(K, x.numel()))
            best += [(-v, w, int(ids[j])) for v, j in zip(top.values.tolist(), top.indices.tolist())]
        best = sorted(best)[:K] + [(float("inf"), -1, -1)] * max(0, K - len(best))
        for v, w, t in best:
            lists[0].append(-v)
            lists[1].append(w)
            lists[2].append(t)
            lists[3].append(w >= 0 and (t == EOS or (s["done"] is not None and bool(s["done"][g, w]))))
    return (torch.tensor(lists[0], dtype=torch.float64, device="cuda").view(G, K), _ints(lists[1]).view(G, K),
            _ints(lists[2]).view(G, K), torch.tensor(lists[3], device="cuda").view(G, K))


def _exact_reorder(s):
    c = s["c"]
    G, W, ps = c["groups"], c["beams"], c["page"]
    table = s["table"].tolist()
    new = [list(r) for r in table]
    ks, vs = [[] for _ in range(c["layers"])], [[] for _ in range(c["layers"])]
    for g in range(G):
        p, x = s["parent"][g].tolist(), s["ctx_len"][g * W].item()
        free = [b for b in range(W) if b not in p]
        for b in range(W):
            new[g * W + b][:x // ps] = table[g * W + p[b]][:x // ps]
            if x % ps:
                new[g * W + b][x // ps] = table[g * W + (p[b] if p[b] not in p[:b] else free.pop(0))][x // ps]
            for i in range(c["layers"]):
                k, v = _read64(s, i, g * W + p[b], torch.arange(x - x % ps, x, device="cuda"))
                ks[i].append(k)
                vs[i].append(v)
    return (_ints(new), torch.stack([torch.cat(x) for x in ks]), torch.stack([torch.cat(x) for x in vs]))
