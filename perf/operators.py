"""Timed cases of the paged KV cache's operators, through the public entry points: kv_append,
kv_read, attn_chunk and verify_draft.

A paged cache holds one layer's keys and values in pages of `page` positions; a table row per
sequence names its pages.  A chunk is a ragged batch of new tokens: sequence b's new rows are
row_start[b] .. row_start[b + 1] - 1, at positions ctx_len[b], ctx_len[b] + 1, ...

    append  rotate q and k (bf16 caches; the keys of int8 cases arrive rotated), write k and v
            to the pages (int8: s = fp16(absmax / 127), code = rint(x / s), per position and
            kv head), then read the new rows back
    read    keys and values of whole sequences as bf16 rows
    attn    softmax(scale q K^T) V, causal: a row at position p sees positions 0 .. p
    verify  accept drafted tokens against the target's logits, one token drawn at the end

Layouts: keys [pages, kv heads, page, d], values [pages, kv heads, page / 32, d, 32] with
position t of a block of 32 in slot 8 ((t % 16) / 4) + 4 (t / 16) + t % 4, int8 scales fp16
[pages, kv heads, page].
"""
import math

import torch

own = False

VOCAB = 32000
BLK = 32
SLOT = [8 * ((t & 15) >> 2) + 4 * (t >> 4) + (t & 3) for t in range(BLK)]


def _attn(name, heads, kv_heads, d, kvq, page, B, ctx, new, mixed=0):
    c = {"kind": "attn", "heads": heads, "kv_heads": kv_heads, "d": d, "kvq": kvq, "page": page, "B": B,
         "ctx": ctx, "new": new, "mixed": mixed}
    return c if name is None else dict(c, name=name)


def _append(name, heads, kv_heads, d, kvq, page, B, ctx, new):
    return dict(_attn(name, heads, kv_heads, d, kvq, page, B, ctx, new), kind="append")


def _read(name, kv_heads, d, kvq, page, B, length):
    return dict(_attn(name, 0, kv_heads, d, kvq, page, B, 0, length), kind="read")


def _verify(name, B, drafts, vocab, probs, temperature):
    c = {"kind": "verify", "B": B, "drafts": drafts, "vocab": vocab, "probs": probs, "temperature": temperature}
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one user's next token over a short context: the smallest call, latency
        _attn("attn-one-token", 32, 32, 128, "bf16", 64, 1, 331, 1),
        # a serving batch's next tokens, contexts of all lengths, grouped queries, int8 cache
        _attn("attn-batch-token", 64, 8, 128, "int8", 64, 32, 16384, 1),
        # four drafted tokens per sequence, checked in one pass
        _attn("attn-drafts", 32, 4, 128, "bf16", 32, 16, 4000, 5),
        # an ordinary chunk of a long prompt (7B shape)
        _attn("attn-chunk", 32, 32, 128, "bf16", 128, 1, 1536, 512),
        # a large chunk far into a long prompt, 70B tensor-parallel shard, int8 cache
        _attn("attn-long-chunk", 8, 1, 128, "int8", 256, 1, 30001, 2048),
        # one prompt's chunk in a batch of next tokens, odd sizes, head_dim 64
        _attn("attn-mixed", 24, 6, 64, "bf16", 96, 17, 1777, 1000, mixed=16),
        # a batch's next tokens enter an int8 cache
        _append("append-tokens", 64, 8, 128, "int8", 64, 64, 3000, 1),
        # the chunks of several prompts enter a bf16 cache, queries and keys rotated
        _append("append-chunks", 32, 8, 128, "bf16", 128, 5, 4001, 2048),
        # short sequences leave the cache (a preempted request), odd sizes
        _read("read-short", 6, 64, "int8", 32, 5, 333),
        # a batch of long int8 sequences read back as bf16
        _read("read-long", 8, 128, "int8", 64, 8, 16000),
        # one sequence's three drafted tokens against greedy target decoding
        _verify("verify-one", 1, 3, VOCAB, False, 0.0),
        # a batch's drafts with the draft model's probabilities
        _verify("verify-batch", 32, 5, VOCAB, True, 0.8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """A case of the same ranges: kv heads 1 to 32 with 1 to 16 query heads each, head_dim 64 or
    128, either cache format, pages of 32 to 256 positions, 1 to 64 sequences of 1 to 32768
    positions, chunks of 1 to 2048 tokens; vocabularies of 1000 to 160000 ids and 0 to 8 drafts."""
    top_b = max(work(c)["bytes"] for c in listed())
    top_f = max(work(c)["flops"] for c in listed())
    while True:
        kind = rng.choice(["attn", "attn", "attn", "append", "read", "verify"])
        if kind == "verify":
            c = _verify(None, _log(rng, 1, 64), rng.randint(0, 8), _log(rng, 1000, 160000), rng.random() < 0.6,
                        rng.choice([0.0, 0.5, 0.7, 1.0, 1.3]))
        else:
            nkv, g, d = rng.choice([1, 2, 3, 4, 6, 8, 16, 32]), rng.choice([1, 1, 2, 3, 4, 5, 8, 16]), rng.choice([64, 128])
            kvq, page, B = rng.choice(["bf16", "int8"]), 32 * rng.randint(1, 8), _log(rng, 1, 64)
            ctx = _log(rng, 1, 32768) - 1
            new = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 1, 2048)])
            if kind == "attn":
                mixed = rng.randint(1, 32) if rng.random() < 0.25 else 0
                c = _attn(None, nkv * g, nkv, d, kvq, page, B + mixed, ctx, new, mixed)
            elif kind == "append":
                c = _append(None, nkv * g, nkv, d, kvq, page, B, ctx, new)
            else:
                c = _read(None, nkv, d, kvq, page, B, ctx + 1)
            if c["heads"] > 128:
                continue
        w = work(c)
        pool = 0 if kind == "verify" else c["B"] * (c["ctx"] + c["new"] + c["page"]) * c["kv_heads"] * c["d"] * 4
        if w["bytes"] <= top_b and w["flops"] <= top_f and pool <= 4 << 30:
            return c


# ------------------------------------------------------------------ lengths
def _lengths(c):
    """(context, new) of each sequence: the last one has the full context and chunk, the others
    a spread below it (the first `mixed` sequences have one new token)."""
    out = []
    for b in range(c["B"]):
        last = b == c["B"] - 1
        f = 1.0 if last else ((b * 7919 + 5) % 97) / 97.0
        ctx, new = int(c["ctx"] * f), c["new"]
        if not last and new > 16:
            new = max(1, int(new * (0.25 + 0.75 * f)))
        if b < c["mixed"]:
            new = 1
        if c["kind"] == "read":
            ctx, new = 0, max(1, int(c["new"] * f))
        out.append((ctx, new))
    return out


def work(c):
    """Bytes and operations of one pass: every input read once, every output written once."""
    if c["kind"] == "verify":
        rows, B = c["B"] * (c["drafts"] + 1), c["B"]
        b = 4.0 * rows * c["vocab"] + 12.0 * rows + 8.0 * B
        if c["probs"] and c["temperature"] > 0 and c["drafts"] > 0:
            b += 4.0 * B * c["vocab"]
        return {"bytes": b, "flops": 4.0 * rows * c["vocab"]}
    L = _lengths(c)
    nkv, d, H = c["kv_heads"], c["d"], c["heads"]
    per = nkv * (2 * d * (1 if c["kvq"] == "int8" else 2) + (4 if c["kvq"] == "int8" else 0))
    new, total = sum(n for _, n in L), sum(x + n for x, n in L)
    if c["kind"] == "read":
        return {"bytes": float(total * (per + 4 * nkv * d)), "flops": float(2 * total * nkv * d)}
    if c["kind"] == "append":
        # k and v in, the cache out, the new rows read back; queries in and out
        b = new * (4 * nkv * d + 2 * per + 4 * nkv * d)
        f = 6 * new * nkv * d
        if c["kvq"] == "bf16":
            b += new * 4 * H * d + new * 4 * d
            f += 3 * new * H * d
        return {"bytes": float(b), "flops": float(f)}
    pairs = sum(n * x + n * (n + 1) // 2 for x, n in L)
    return {"bytes": float(total * per + new * 4 * H * d), "flops": 4.0 * d * H * pairs}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) % (1 << 62))


def _quantise(x):
    """x [..., d] -> int8 codes and fp16 scales [...]."""
    s = (x.abs().amax(-1) / 127.0).half()
    q = torch.where(s[..., None] > 0, x / s[..., None].float(), torch.zeros_like(x))
    return q.round().clamp(-127, 127).to(torch.int8), s


def _angles(n, d):
    inv = 1e4 ** (-torch.arange(d // 2, device="cuda", dtype=torch.float64) * 2.0 / d)
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


def prepare(c, seed):
    g = _gen(seed)
    dev = torch.device("cuda")
    if c["kind"] == "verify":
        return _prepare_verify(c, g)
    L = _lengths(c)
    nkv, d, H, ps, B = c["kv_heads"], c["d"], c["heads"], c["page"], c["B"]
    lens = [x + n for x, n in L]
    need = [-(-n // ps) for n in lens]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=g, device=dev).int()
    table = torch.full((B, max(need)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    starts = [0]
    for _, n in L:
        starts.append(starts[-1] + n)
    N = starts[-1]
    s = {"c": c, "L": L, "starts": starts, "table": table,
         "row_start": torch.tensor(starts, dtype=torch.int32, device=dev),
         "ctx_len": torch.tensor([x for x, _ in L], dtype=torch.int32, device=dev)}
    # pages as earlier steps left them: every position holds some token's key and value
    chan = torch.exp(0.4 * torch.randn(nkv, 1, d, generator=g, device=dev))
    pool = {}
    for name in ("k", "v"):
        x = torch.randn(n_pages, nkv, ps, d, generator=g, device=dev) * chan
        if name == "k":
            x /= chan.pow(2).mean().sqrt()
        if c["kvq"] == "int8":
            x, pool[name + "_scales"] = _quantise(x)
        else:
            x = x.bfloat16()
        if name == "v":
            y = torch.empty(n_pages, nkv, ps // BLK, d, BLK, dtype=x.dtype, device=dev)
            y[..., torch.tensor(SLOT, device=dev)] = x.view(n_pages, nkv, ps // BLK, BLK, d).transpose(-1, -2)
            x = y
        pool[name] = x
    s["pool"] = pool
    if c["kind"] == "attn":
        s["q"] = (1.5 * torch.randn(N, H, d, generator=g, device=dev)).bfloat16()
        s["out"] = torch.empty(N, H, d, dtype=torch.bfloat16, device=dev)
    elif c["kind"] == "append":
        # the columns of one fused projection's output
        qkv = torch.randn(N, H + 2 * nkv, d, generator=g, device=dev).bfloat16()
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + nkv], qkv[:, H + nkv:]
        s["cos"], s["sin"] = _angles(max(lens), d)
        s["q_out"] = torch.empty(N, H, d, dtype=torch.bfloat16, device=dev)
    if c["kind"] != "attn":
        s["k_out"] = torch.empty(N, nkv, d, dtype=torch.bfloat16, device=dev)
        s["v_out"] = torch.empty(N, nkv, d, dtype=torch.bfloat16, device=dev)
    if own:
        import paper_2501_13111_amd as fp
        s["kv"] = fp.PagedKV(**pool)
        s["chunk"] = fp.Chunk(s["row_start"], s["ctx_len"], table, max_new=max(n for _, n in L), max_len=max(lens))
        if c["kind"] == "attn":
            s["workspace"] = fp.attn_chunk_workspace(s["kv"], s["chunk"], N, H)
    return s


def _prepare_verify(c, g):
    dev = torch.device("cuda")
    B, R, V = c["B"], c["drafts"] + 1, c["vocab"]
    N = B * R
    logits = 2.5 * torch.randn(N, V, generator=g, device=dev)
    # a few likely tokens per row, and a draft that mostly agrees with the target
    logits.scatter_add_(1, torch.randint(V, (N, 8), generator=g, device=dev), 9 * torch.rand(N, 8, generator=g, device=dev))
    T = c["temperature"]
    noisy = logits + 0.5 * torch.randn(N, V, generator=g, device=dev)
    if T > 0 and c["probs"]:
        probs = torch.softmax(noisy.double() / T, -1).float()
        pick = torch.rand(N, 1, generator=g, device=dev, dtype=torch.float64)
        ids = (probs.double().cumsum(-1) <= pick).sum(-1).clamp_(max=V - 1).int()
    else:
        probs = None
        ids = noisy.argmax(-1).int()
    s = {"c": c, "logits": logits, "ids": ids, "probs": probs,
         "row_start": torch.arange(0, N + 1, R, dtype=torch.int32, device=dev),
         "u": torch.rand(N, generator=g, device=dev), "u_last": torch.rand(B, generator=g, device=dev),
         "out_ids": torch.empty(B, R, dtype=torch.int32, device=dev),
         "n_out": torch.empty(B, dtype=torch.int32, device=dev)}
    if own:
        import paper_2501_13111_amd as fp
        s["workspace"] = fp.verify_draft_workspace(N, V)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    if own:
        import paper_2501_13111_amd as fp
        if c["kind"] == "attn":
            fp.attn_chunk(s["kv"], s["chunk"], s["q"], s["out"], workspace=s["workspace"])
            return s["out"]
        if c["kind"] == "read":
            fp.kv_read(s["kv"], s["chunk"], s["k_out"], s["v_out"])
            return s["k_out"], s["v_out"]
        if c["kind"] == "append":
            if c["kvq"] == "bf16":
                fp.kv_append(s["kv"], s["chunk"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], cos=s["cos"], sin=s["sin"])
                fp.kv_read(s["kv"], s["chunk"], s["k_out"], s["v_out"])
                return s["q_out"], s["k_out"], s["v_out"]
            fp.kv_append(s["kv"], s["chunk"], s["k"], s["v"])
            fp.kv_read(s["kv"], s["chunk"], s["k_out"], s["v_out"])
            return s["k_out"], s["v_out"]
        fp.verify_draft(s["logits"], s["row_start"], s["ids"], s["u"], s["u_last"], s["out_ids"], s["n_out"],
                        draft_probs=s["probs"], temperature=c["temperature"], workspace=s["workspace"])
        return s["out_ids"], s["n_out"]
    return {"attn": _plain_attn, "read": _plain_read, "append": _plain_append, "verify": _plain_verify}[c["kind"]](s)


def _sequence(s, b, length):
    """Keys and values of positions 0 .. length - 1 of sequence b, fp32 [length, kv heads, d]."""
    c, pool = s["c"], s["pool"]
    ps, nkv, d = c["page"], c["kv_heads"], c["d"]
    pages = s["table"][b, :-(-length // ps)].long()
    k = pool["k"][pages].float()
    v = pool["v"][pages][..., torch.tensor(SLOT, device="cuda")].float().transpose(-1, -2).reshape(-1, nkv, ps, d)
    if c["kvq"] == "int8":
        k = k * pool["k_scales"][pages].float()[..., None]
        v = v * pool["v_scales"][pages].float()[..., None]
    return (k.transpose(1, 2).reshape(-1, nkv, d)[:length], v.transpose(1, 2).reshape(-1, nkv, d)[:length])


def _plain_attn(s):
    c = s["c"]
    H, nkv, d = c["heads"], c["kv_heads"], c["d"]
    G = H // nkv
    out = s["out"]
    for b, (ctx, new) in enumerate(s["L"]):
        n = ctx + new
        k, v = _sequence(s, b, n)
        kt = k.permute(1, 2, 0).contiguous()                                # [kv heads, d, n]
        vh = v.transpose(0, 1).contiguous()                                 # [kv heads, n, d]
        step = max(1, (1 << 28) // (H * n))
        for r0 in range(0, new, step):
            r1 = min(new, r0 + step)
            rows = slice(s["starts"][b] + r0, s["starts"][b] + r1)
            q = s["q"][rows].float().view(r1 - r0, nkv, G, d).permute(1, 0, 2, 3).reshape(nkv, -1, d)
            sc = torch.bmm(q, kt) * (1.0 / math.sqrt(d))
            pos = torch.arange(ctx + r0, ctx + r1, device="cuda").repeat_interleave(G)
            sc.masked_fill_(torch.arange(n, device="cuda")[None, :] > pos[:, None], float("-inf"))
            e = torch.exp(sc - sc.amax(-1, keepdim=True))
            o = torch.bmm(e, vh) / e.sum(-1, keepdim=True)
            out[rows] = o.view(nkv, r1 - r0, G, d).permute(1, 0, 2, 3).reshape(r1 - r0, H, d).bfloat16()
    return out


def _plain_read(s):
    for b, (_, n) in enumerate(s["L"]):
        rows = slice(s["starts"][b], s["starts"][b + 1])
        k, v = _sequence(s, b, n)
        s["k_out"][rows] = k.bfloat16()
        s["v_out"][rows] = v.bfloat16()
    return s["k_out"], s["v_out"]


def _plain_append(s):
    c, pool = s["c"], s["pool"]
    ps, d = c["page"], c["d"]
    new = torch.tensor([n for _, n in s["L"]], device="cuda")
    seq = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), new, output_size=s["starts"][-1])
    row = torch.arange(s["starts"][-1], device="cuda")
    pos = s["ctx_len"].long()[seq] + row - s["row_start"].long()[seq]
    page, off = s["table"][seq, pos // ps].long(), pos % ps
    k, v = s["k"].float(), s["v"].float()
    if c["kvq"] == "bf16":
        cos, sin = s["cos"][pos][:, None, :], s["sin"][pos][:, None, :]

        def rotate(x):
            lo, hi = x[..., :d // 2], x[..., d // 2:]
            return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

        s["q_out"].copy_(rotate(s["q"].float()).bfloat16())
        k, v = rotate(k).bfloat16(), v.bfloat16()
        ks = vs = None
    else:
        k, ks = _quantise(k)
        v, vs = _quantise(v)
        pool["k_scales"][page, :, off] = ks
        pool["v_scales"][page, :, off] = vs
    slot = torch.tensor(SLOT, device="cuda")[off % BLK]
    pool["k"][page, :, off] = k
    pool["v"][page, :, off // BLK, :, slot] = v
    kb, vb = pool["k"][page, :, off].float(), pool["v"][page, :, off // BLK, :, slot].float()
    if ks is not None:
        kb = kb * pool["k_scales"][page, :, off].float()[..., None]
        vb = vb * pool["v_scales"][page, :, off].float()[..., None]
    s["k_out"].copy_(kb.bfloat16())
    s["v_out"].copy_(vb.bfloat16())
    return (s["q_out"], s["k_out"], s["v_out"]) if ks is None else (s["k_out"], s["v_out"])


def _plain_verify(s):
    """All rows at once, in 64 bits: the borders of the draws decide."""
    c = s["c"]
    B, R, V, T = c["B"], c["drafts"] + 1, c["vocab"], c["temperature"]
    ids = s["ids"].long()
    if T == 0:
        best = s["logits"].argmax(-1)
        ok = ids == best
    else:
        z = s["logits"].double() / T
        e = torch.exp(z - z.amax(-1, keepdim=True))
        p = e / e.sum(-1, keepdim=True)
        at = p.gather(1, ids[:, None])[:, 0]
        q = s["probs"].gather(1, ids[:, None])[:, 0].double() if s["probs"] is not None else torch.ones_like(at)
        ok = s["u"].double() * q < at
    acc = ok.view(B, R)[:, :R - 1].long().cumprod(-1).sum(-1)               # drafts accepted in a row
    row = torch.arange(B, device="cuda") * R + acc
    if T == 0:
        last = best[row]
    else:
        res = p[row]
        bonus = (acc == R - 1)[:, None]
        if s["probs"] is not None:
            res = torch.where(bonus, res, (res - s["probs"][row].double()).clamp(min=0))
        else:
            hit = torch.arange(V, device="cuda")[None, :] == ids[row][:, None]
            res = torch.where(hit & ~bonus, torch.zeros_like(res), res)
        res = torch.where(res.sum(-1, keepdim=True) > 0, res, p[row])
        cum = res.cumsum(-1)
        last = (cum <= s["u_last"].double()[:, None] * cum[:, -1:]).sum(-1)
        top = torch.where(res > 0, torch.arange(V, device="cuda")[None, :], torch.zeros_like(res, dtype=torch.long)).amax(-1)
        last = torch.minimum(last, top)
    j = torch.arange(R, device="cuda")[None, :]
    out = torch.where(j < acc[:, None], ids.view(B, R), torch.full_like(j, -1))
    out = torch.where(j == acc[:, None], last[:, None], out)
    s["out_ids"].copy_(out)
    s["n_out"].copy_(acc + 1)
    return s["out_ids"], s["n_out"]


# ------------------------------------------------------------------ 64 bits, from the definitions
def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "verify":
        return _exact_verify(s)
    dev = "cuda"
    ps, nkv, d, H = c["page"], c["kv_heads"], c["d"], c["heads"]
    slot = torch.tensor(SLOT, device=dev)

    def cached(b, p):
        """Keys and values at positions p of sequence b, [positions, kv heads, d]."""
        pg, off = s["table"][b].long()[p // ps], p % ps
        k, v = s["pool"]["k"][pg, :, off].double(), s["pool"]["v"][pg, :, off // BLK, :, slot[off % BLK]].double()
        if c["kvq"] == "int8":
            k = k * s["pool"]["k_scales"][pg, :, off].double()[..., None]
            v = v * s["pool"]["v_scales"][pg, :, off].double()[..., None]
        return k, v

    if c["kind"] == "read":
        ks, vs = zip(*(cached(b, torch.arange(n, device=dev)) for b, (_, n) in enumerate(s["L"])))
        return torch.cat(ks), torch.cat(vs)
    if c["kind"] == "append":
        k, v = s["k"].double(), s["v"].double()
        if c["kvq"] == "int8":
            def held(x):
                # the scale is an fp16 number by definition, the codes are whole numbers
                sc = (x.abs().amax(-1) / 127.0).half().double()[..., None]
                return torch.where(sc > 0, (x / sc).round().clamp(-127, 127) * sc, torch.zeros_like(x))
            return held(k), held(v)
        pos = torch.cat([torch.arange(x, x + n, device=dev) for x, n in s["L"]])
        cos, sin = s["cos"].double()[pos], s["sin"].double()[pos]
        turn = torch.complex(cos, sin)[:, None, :]

        def rot(x):
            z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)
        return rot(s["q"].double()), rot(k), v
    G = H // nkv
    out = torch.empty(s["starts"][-1], H, d, dtype=torch.float64, device=dev)
    for b, (ctx, new) in enumerate(s["L"]):
        n = ctx + new
        k, v = cached(b, torch.arange(n, device=dev))
        q = s["q"][s["starts"][b]:s["starts"][b + 1]].double()
        step = max(1, (1 << 26) // (n * G))
        for h in range(nkv):
            kh, vh = k[:, h].t().contiguous(), v[:, h].contiguous()
            for r0 in range(0, new, step):
                qh = q[r0:r0 + step, h * G:(h + 1) * G]
                m = qh.shape[0]
                sc = (qh.reshape(m * G, d) @ kh).view(m, G, n) / math.sqrt(d)
                seen = torch.arange(n, device=dev)[None, :] <= torch.arange(ctx + r0, ctx + r0 + m, device=dev)[:, None]
                sc = torch.where(seen[:, None, :], sc, torch.full_like(sc, float("-inf")))
                p = torch.softmax(sc, -1)
                at = s["starts"][b] + r0
                out[at:at + m, h * G:(h + 1) * G] = (p.view(m * G, n) @ vh).view(m, G, d)
    return out


def _exact_verify(s):
    """One sequence and one row after another."""
    c = s["c"]
    R, T = c["drafts"] + 1, c["temperature"]
    ids, u, ul = s["ids"].tolist(), s["u"].tolist(), s["u_last"].tolist()
    out = torch.full((c["B"], R), -1, dtype=torch.int32)
    count = torch.zeros(c["B"], dtype=torch.int32)
    for b in range(c["B"]):
        for i in range(R):
            r = b * R + i
            x = s["logits"][r].double()
            drafted = i < R - 1
            if T == 0:
                best = int((x == x.max()).nonzero()[0])
                out[b, i] = best
                count[b] = i + 1
                if drafted and ids[r] == best:
                    continue
                break
            p = torch.softmax(x / T, -1)
            if drafted:
                q = s["probs"][r].double() if s["probs"] is not None else None
                qx = 1.0 if q is None else float(q[ids[r]])
                if u[r] * qx < float(p[ids[r]]):
                    out[b, i] = ids[r]
                    continue
                if q is None:
                    left = p.clone()
                    left[ids[r]] = 0.0
                else:
                    left = (p - q).clamp(min=0)
                if float(left.sum()) > 0:
                    p = left
            cum = p.cumsum(-1)
            above = (cum > ul[b] * cum[-1]).nonzero()
            out[b, i] = int(above[0]) if len(above) else int(p.nonzero()[-1])
            count[b] = i + 1
            break
    return out.cuda(), count.cuda()
