"""Plain 64-bit reference of drafted trees and beams on a paged cache (test infrastructure; loops where they are
clearest)."""
import math

import torch


def lines(parent):
    """Of each node of one sequence the nodes from the root down to it; a parent that is no earlier node is none."""
    out = []
    for i, p in enumerate(parent):
        out.append((out[p] if 0 <= p < i else []) + [i])
    return out


def random_tree(g, n, forest=False):
    """Parents of n nodes; forest: some hang on nothing, and some name nodes that they may not."""
    p = [-1] + [int(torch.randint(0, i, (1,), generator=g)) for i in range(1, n)]
    if forest:
        junk = [-1, -7, n, 2**31 - 1, -(2**31)]
        for i in range(1, n):
            if torch.rand(1, generator=g) < 0.25:
                p[i] = (junk + [i, i + 1])[int(torch.randint(0, len(junk) + 2, (1,), generator=g))]
    return p


def tree_attention(pool, table, lens, parent, q, scale=None):
    """As paged_reference.attention, where row i of a sequence sees its context and its line."""
    H, d = q.shape[1], q.shape[2]
    G = H // pool.nkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, mag, smag = (torch.zeros(q.shape[0], H, d, dtype=torch.float64) for _ in range(3))
    r = 0
    for b, (ctx, new) in enumerate(lens):
        if new == 0:
            continue
        k, v = pool.read(table[b], ctx + new)
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        for i, line in enumerate(lines(parent[r:r + new])):
            at = torch.cat([torch.arange(ctx), ctx + torch.tensor(line)])
            qq, kk, vv = q[r + i].double(), k[at], v[at]
            s = torch.einsum("hd,nhd->hn", qq, kk) * scale
            p = torch.softmax(s, -1)
            out[r + i] = torch.einsum("hn,nhd->hd", p, vv)
            mag[r + i] = torch.einsum("hn,nhd->hd", p, vv.abs())
            smag[r + i] = (torch.einsum("hd,nhd->hn", qq.abs(), kk.abs()) * abs(scale)).amax(-1)[:, None]
        r += new
    return out, mag, smag


def verify_tree(logits, row_start, parent, ids, u, T, max_rows):
    """Per sequence (tokens, nodes)."""
    res = []
    for b in range(len(row_start) - 1):
        r0, n = row_start[b], min(row_start[b + 1] - row_start[b], max_rows)
        toks, path, i = [], [], 0
        while n:
            z = logits[r0 + i].double()
            z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
            m = float(z.max())
            if m == -math.inf:
                y = -1
            elif T == 0:
                y = int((z == m).nonzero()[0])
            else:
                w = (z == m).double() if m == math.inf else torch.exp((z - m) / T)
                c = w.cumsum(0)
                above = ((c > float(u[r0 + i]) * c[-1]) & (w > 0)).nonzero()
                y = int(above[0]) if len(above) else int((w > 0).nonzero()[-1])
            toks.append(y)
            path.append(i)
            nxt = [j for j in range(i + 1, n) if parent[r0 + j] == i and ids[r0 + j] == y and y >= 0]
            if not nxt:
                break
            i = nxt[0]
        res.append((toks, path))
    return res


def beam_select(logits, scores, done, K, eos, pad):
    """Per group K tuples (score, parent, id, done): logits [G, W, V], scores [G, W] -> lists."""
    G, W, V = logits.shape
    res = []
    for g in range(G):
        cand = []
        for w in range(W):
            s = float(scores[g, w])
            if math.isnan(s) or s == -math.inf:
                continue
            if done is not None and done[g, w]:
                cand.append((-s, w, 0.0, pad, True))
                continue
            z = logits[g, w].double()
            z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
            m = float(z.max())
            if m == -math.inf:
                continue
            if m == math.inf:
                base, on = s - math.log(float((z == m).sum())), z == m
                sc = torch.where(on, torch.full_like(z, base), torch.full_like(z, -math.inf))
            else:
                sc, on = (s - math.log(float(torch.exp(z - m).sum()))) + (z - m), z > -math.inf
            ids = on.nonzero()[:, 0]
            # the largest K by (logit, lower id)
            order = sorted(((-float(z[v]), int(v)) for v in (ids[torch.argsort(-z[ids], stable=True)][:K])))
            cand += [(-float(sc[v]), w, nz, v, v == eos) for nz, v in order]
        cand = sorted(cand)[:K]
        res.append([(-c[0], c[1], c[3], c[4]) for c in cand] + [(-math.inf, -1, -1, False)] * (K - len(cand)))
    return res


def reorder(table, length, parent, page, n_beams):
    """One group's rows -> (new rows, [(from page, to page)] of the last pages' copies)."""
    W = n_beams
    p = [x if 0 <= x < W else b for b, x in enumerate(parent)]
    new, copies = [list(r) for r in table], []
    full, part = length // page, length % page
    free = [b for b in range(W) if b not in p]
    for b in range(W):
        new[b][:full] = table[p[b]][:full]
        if part and full < len(new[b]):
            if p[b] in p[:b]:
                new[b][full] = table[free.pop(0)][full]
                copies.append((table[p[b]][full], new[b][full]))
            else:
                new[b][full] = table[p[b]][full]
    return new, copies
