"""Plain 64-bit reference of the paged cache, the attention of a chunk over it and the
verification of drafts (test infrastructure; torch on the CPU, loops where they are clearest)."""
import math

import torch

BLK = 32
SLOT = torch.tensor([8 * ((t % 16) // 4) + 4 * (t // 16) + t % 4 for t in range(BLK)])


def bits(t):
    return t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


class Pool:
    """A pool whose unwritten positions hold NaN (bf16), or codes of -128 and NaN scales (int8)."""

    def __init__(self, n_pages, page, nkv, d, kvq):
        self.page, self.nkv, self.d, self.kvq, self.n_pages = page, nkv, d, kvq, n_pages
        if kvq == "int8":
            self.k = torch.full((n_pages, nkv, page, d), -128, dtype=torch.int8)
            self.v = torch.full((n_pages, nkv, page // BLK, d, BLK), -128, dtype=torch.int8)
            self.ks = torch.full((n_pages, nkv, page), math.nan, dtype=torch.float16)
            self.vs = self.ks.clone()
        else:
            self.k = torch.full((n_pages, nkv, page, d), math.nan, dtype=torch.bfloat16)
            self.v = torch.full((n_pages, nkv, page // BLK, d, BLK), math.nan, dtype=torch.bfloat16)
            self.ks = self.vs = None

    def tensors(self):
        return [self.k, self.v] + ([self.ks, self.vs] if self.kvq == "int8" else [])

    def device(self):
        import paper_2501_13111_amd as fp
        return fp.PagedKV(*[t.cuda() for t in self.tensors()])

    def _at(self, table, pos):
        pages = table[torch.as_tensor(pos) // self.page].long()
        return pages, torch.as_tensor(pos) % self.page

    def write(self, table, pos, k, v):
        """k, v float32 [positions, nkv, d], already rotated, into the positions pos."""
        pg, off = self._at(table, pos)
        if self.kvq == "int8":
            k, self.ks[pg, :, off] = quantise(k)
            v, self.vs[pg, :, off] = quantise(v)
        else:
            k, v = k.bfloat16(), v.bfloat16()
        self.k[pg, :, off] = k
        self.v[pg, :, off // BLK, :, SLOT[off % BLK]] = v

    def read(self, table, n):
        """Positions 0 .. n - 1 as float64 [n, nkv, d] (missing pages: zeros)."""
        pos = torch.arange(n)
        pg, off = self._at(table, pos)
        bad = (pg < 0) | (pg >= self.n_pages)
        pg = torch.where(bad, torch.zeros_like(pg), pg)
        k, v = self.k[pg, :, off].double(), self.v[pg, :, off // BLK, :, SLOT[off % BLK]].double()
        if self.kvq == "int8":
            k = k * self.ks[pg, :, off].double()[..., None]
            v = v * self.vs[pg, :, off].double()[..., None]
        k[bad] = 0.0
        v[bad] = 0.0
        return k, v


def quantise(x):
    """float32 [..., d] -> int8 codes, fp16 scales: the cache's rule in fp32."""
    s = (x.abs().amax(-1) / 127.0).half()
    sf = s.float()[..., None]
    c = torch.where(sf > 0, (x / torch.where(sf > 0, sf, torch.ones_like(sf))).round(), torch.zeros_like(x))
    return c.clamp(-127, 127).to(torch.int8), s


def tables(g, need, n_pages, width, junk=(-1, 2**30, -(2**31))):
    """A page table with every page used once, in random order; entries past a sequence's pages
    are junk."""
    perm = torch.randperm(n_pages, generator=g)
    t = torch.zeros(len(need), width, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = perm[at:at + n].int()
        for i in range(n, width):
            t[b, i] = junk[(b + i) % len(junk)]
        at += n
    return t


def rope_tables(n, d, theta=1e4):
    inv = theta ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d)
    a = torch.arange(n, dtype=torch.float64)[:, None] * inv
    return a.cos().float(), a.sin().float()


def rotate(x, pos, cos, sin):
    """float64 rotation of x [rows, heads, d] at positions pos, from the float32 tables."""
    h = x.shape[-1] // 2
    c, s = cos.double()[pos][:, None, :], sin.double()[pos][:, None, :]
    lo, hi = x[..., :h].double(), x[..., h:].double()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def attention(pool, table, lens, q, scale=None):
    """q [rows, H, d] of the ragged sequences lens = [(ctx, new)] -> (out, sum of p |v|, largest
    |q| |k| scale sum of a row), all float64."""
    H, d = q.shape[1], q.shape[2]
    G = H // pool.nkv
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, mag, smag = (torch.zeros(q.shape[0], H, d, dtype=torch.float64) for _ in range(3))
    r = 0
    for b, (ctx, new) in enumerate(lens):
        if new == 0:
            continue
        k, v = pool.read(table[b], ctx + new)
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)           # [n, H, d]
        qq = q[r:r + new].double()
        for i in range(new):
            n = ctx + i + 1
            s = torch.einsum("hd,nhd->hn", qq[i], k[:n]) * scale
            p = torch.softmax(s, -1)
            out[r + i] = torch.einsum("hn,nhd->hd", p, v[:n])
            mag[r + i] = torch.einsum("hn,nhd->hd", p, v[:n].abs())
            smag[r + i] = (torch.einsum("hd,nhd->hn", qq[i].abs(), k[:n].abs()) * abs(scale)).amax(-1)[:, None]
        r += new
    return out, mag, smag


def verify(logits, row_start, draft_ids, probs, u, u_last, T, max_rows):
    """Lists of tokens per sequence, row by row in float64."""
    V = logits.shape[1]
    res = []
    for b in range(len(row_start) - 1):
        rows = list(range(row_start[b], row_start[b + 1]))[:max_rows]
        toks = []
        for i, r in enumerate(rows):
            z = logits[r].double()
            z = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
            x = int(draft_ids[r]) if i < len(rows) - 1 else None
            m = float(z.max())
            if m == -math.inf:
                toks.append(-1)
                break
            first = int((z == m).nonzero()[0])
            if T == 0:
                if x is not None and x == first:
                    toks.append(x)
                    continue
                toks.append(first)
                break
            e = (z == m).double() if m == math.inf else torch.exp((z - m) / T)
            p = e / e.sum()
            w = p
            if x is not None:
                q = None if probs is None else torch.nan_to_num(probs[r].double(), nan=0.0).clamp(min=0)
                inside = 0 <= x < V
                if inside:
                    qx = 1.0 if q is None else float(q[x])
                    if float(u[r]) * qx < float(p[x]):
                        toks.append(x)
                        continue
                if q is None:
                    w = p.clone()
                    if inside:
                        w[x] = 0
                else:
                    w = (p - q).clamp(min=0)
                if not float(w.sum()) > 0:
                    w = p
            c = w.cumsum(0)
            above = ((c > float(u_last[b]) * c[-1]) & (w > 0)).nonzero()
            toks.append(int(above[0]) if len(above) else int((w > 0).nonzero()[-1]))
            break
        res.append(toks)
    return res
