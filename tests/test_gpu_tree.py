"""Drafted trees on the GPU against plain 64-bit references: attention over a paged cache, the append's rotation by depth,
verification, the accepted path's move, the layer stack, and a run of them together."""
import math

import numpy as np
import pytest
import torch

import branches_reference as bref
import paged_reference as ref
import test_gpu_paged as paged
from fpgen.workloads import Shape
from test_gpu_extend import Paged
from tests.gpu_harness import TOL, bf16_to_np, np_to_bf16, rel_inf

pytestmark = pytest.mark.gpu

HALF_BF16, EPS32 = paged.HALF_BF16, paged.EPS32
_fp = paged._fp


def _trees(g, lens, forest=False):
    return sum([bref.random_tree(g, n, forest) for _, n in lens if n], [])


def _int(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _check(pool, table, lens, parent, q, out, scale=None, fp16=False, floor=0.0):
    """The bound of the chunk attention's test (output's rounding, probabilities rounded before they meet v, fp32 scores)."""
    want, mag, smag = bref.tree_attention(pool, table, lens, parent, q, scale)
    ds = 2 * (q.shape[2] + 4) * EPS32 * smag
    if fp16:
        ds = ds + 2 * 2.0 ** -11 * smag
    tol = HALF_BF16 * want.abs() + (HALF_BF16 + 2 * ds + 1e-5 + (2.0 ** -11 if fp16 else 0.0)) * mag * (1 + HALF_BF16) + floor
    err = (out[:want.shape[0]].cpu().double() - want).abs()
    assert (err <= tol).all(), f"{(err / tol.clamp(min=1e-30)).max():.3f} of the tolerance"


TREES = {
    "one": [(0, 1)],
    "few": [(331, 8)],
    "edge": [(31, 2), (32, 5), (63, 33), (0, 32), (0, 33), (95, 1), (96, 64)],
    "ragged": [(5, 3), (0, 0), (100, 17), (64, 0), (33, 64), (0, 1)],
    "split": [(2500, 6), (3, 1), (1100, 20), (700, 64)],
    "mixed": [(40, 1), (250, 50), (900, 1), (0, 64)],
}
SHAPES = [(1, 1, 64, 32), (2, 4, 128, 64), (3, 5, 128, 96), (2, 16, 64, 32), (1, 8, 128, 256), (2, 2, 64, 128)]


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", SHAPES)
@pytest.mark.parametrize("seqs", sorted(TREES))
def test_attention_matches_the_reference(seqs, nkv, G, d, page, kvq, loose):
    fp = _fp()
    lens = TREES[seqs]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 21)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n, scale=1.5)
    parent = _trees(g, lens, forest=page != 64)
    chunk, starts = paged._chunk(lens, table, loose=page * loose)
    N = starts[-1]
    q = torch.randn(N + 2, nkv * G, d, generator=g).bfloat16()
    out = torch.full((N + 2, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    kv, pp = pool.device(), _int(parent + [0, 0])
    fp.attn_tree(kv, chunk, pp, q.cuda(), out)
    assert (out[N:] == 7.0).all()                                # rows behind the last sequence
    _check(pool, table, lens, parent, q[:N], out)
    again = torch.empty_like(out)
    fp.attn_tree(kv, chunk, pp, q.cuda(), again)
    assert torch.equal(ref.bits(again[:N]), ref.bits(out[:N]))


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("n_seqs,nkv,G,nodes", [(20, 8, 8, 16), (300, 1, 8, 16), (12, 4, 4, 32), (70, 4, 8, 9), (300, 1, 4, 17),
                                                      (24, 3, 8, 40)])
def test_many_short_sequences_with_more_than_64_rows(n_seqs, nkv, G, nodes, kvq):
    """Short contexts: whole tiles of 128 rows, which leave no pieces, and of 32; up to and above 256 sequences.  The workspace is as
    large as asked for and not a byte behind it is written."""
    fp = _fp()
    g = torch.Generator().manual_seed(n_seqs + nodes)
    far = 300 if nodes == 40 else 71                            # (more than 128 rows, above 8 blocks)
    lens = [(int(torch.randint(0, far, (1,), generator=g)), nodes - (b * 7 % 3 if b else 0)) for b in range(n_seqs)]
    gg, pool, table = paged._case(lens, 32, nkv, 128, kvq, 23)
    paged._fill(pool, table, lens, gg, upto=lambda c, n: c + n)
    parent = _trees(g, lens)
    chunk, starts = paged._chunk(lens, table)
    q = torch.randn(starts[-1], nkv * G, 128, generator=g).bfloat16()
    kv, out = pool.device(), torch.empty(q.shape, dtype=torch.bfloat16).cuda()
    n = fp.attn_chunk_workspace(kv, chunk, starts[-1], nkv * G).numel()
    room = torch.full((n + 4096,), 0xAB, dtype=torch.uint8).cuda()
    fp.attn_tree(kv, chunk, _int(parent), q.cuda(), out, workspace=room[:n])
    _check(pool, table, lens, parent, q, out, fp16=kvq == "int8", floor=2.0 ** -25 if kvq == "int8" else 0.0)
    assert (room[n:] == 0xAB).all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,page", [(2, 8, 64), (1, 16, 32), (3, 5, 96), (1, 2, 256)])
@pytest.mark.parametrize("seqs", ["one", "edge", "split", "ragged"])
def test_tiles_of_128_rows(seqs, nkv, G, page, kvq):
    """65 to 128 rows to a kv head of 128 dims, beside sequences with fewer."""
    fp = _fp()
    m, d = 128 // G, 128
    lens = {"one": [(331, m)], "edge": [(31, 2), (32, 5), (63, m), (0, m), (0, m - 1), (95, 1), (96, m), (1, m)],
            "split": [(4500, 6), (3, 1), (2100, m), (1700, m - 2)], "ragged": [(5, 3), (0, 0), (100, m), (64, 0), (33, m - 3), (0, 1)]}[seqs]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 22)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n, scale=1.5)
    parent = _trees(g, lens, forest=G == 8)
    chunk, starts = paged._chunk(lens, table, loose=page)
    N = starts[-1]
    q = torch.randn(N + 2, nkv * G, d, generator=g).bfloat16()
    out = torch.full((N + 2, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    kv, pp = pool.device(), _int(parent + [0, 0])
    for scale in (None, -0.05):
        fp.attn_tree(kv, chunk, pp, q.cuda(), out, scale=scale)
        assert (out[N:] == 7.0).all()
        _check(pool, table, lens, parent, q[:N], out, scale, fp16=kvq == "int8", floor=2.0 ** -25 if kvq == "int8" else 0.0)
    again = torch.empty_like(out)
    fp.attn_tree(kv, chunk, pp, q.cuda(), again, scale=-0.05)
    assert torch.equal(ref.bits(again[:N]), ref.bits(out[:N]))


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("G,new,loose", [(4, 5, 0), (4, 30, 0), (8, 14, 64), (8, 60, 64)])
def test_scores_far_apart_and_rising(G, new, loose, kvq):
    """As the chunk's test: the softmax's reference moves again and again, tiny and large values, a negative scale, large queries.
    (5 rows streamed, then tiles of 64 or 32, 128 and 256.)"""
    fp = _fp()
    nkv, d, page, lens = 2, 128, 64, [(900, new), (333, new)]
    for scale, qs in ((None, 1.0), (-0.05, 1.0), (1e-7, 3e5), (3.0, 0.2), (0.0, 1.0)):
        g, pool, table = paged._case(lens, page, nkv, d, kvq, 41)
        for b, (c, n) in enumerate(lens):
            m = c + n
            ramp = torch.linspace(0.1, 6, m)[:, None, None]
            pool.write(table[b], torch.arange(m), (ramp * (1 + 0.2 * torch.randn(m, nkv, d, generator=g))).bfloat16().float(),
                       (torch.randn(m, nkv, d, generator=g) * (10.0 ** (torch.arange(m) % 5 - 3))[:, None, None]).bfloat16().float())
        parent = _trees(g, lens)
        chunk, starts = paged._chunk(lens, table, loose=loose)
        q = (qs * (0.3 + torch.randn(starts[-1], nkv * G, d, generator=g))).bfloat16()
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        fp.attn_tree(pool.device(), chunk, _int(parent), q.cuda(), out, scale=scale)
        # int8, more than 64 rows: keys and values in fp16, of which the smallest are off by 2^-25; probabilities below 2^-21
        # of the largest by 2^-32 of it, times at most all values' magnitudes
        floor = 0.0
        if kvq == "int8":
            vmax = max(float(pool.read(table[b], c + n)[1].abs().sum(0).max()) for b, (c, n) in enumerate(lens))
            floor = 2.0 ** -25 + 2.0 ** -32 * vmax
        _check(pool, table, lens, parent, q, out, scale, fp16=kvq == "int8" and new * G > 64, floor=floor)


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", [(2, 4, 128, 64), (1, 5, 64, 32)])
def test_a_line_is_a_chunk(nkv, G, d, page, kvq, loose):
    """Node i the child of node i - 1: the same bits as the chunk's append, the same attention up to rounding."""
    fp = _fp()
    lens = [(5, 3), (100, 17), (64, 0), (33, 64), (1500, 40), (0, 1)]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 23)
    paged._fill(pool, table, lens, g)
    chunk, starts = paged._chunk(lens, table, loose=page * loose)
    near, _ = paged._chunk(lens, table)
    N = starts[-1]
    parent = _int(sum([list(range(-1, n - 1)) for _, n in lens], []))
    cos, sin = (t.cuda() for t in ref.rope_tables(1600, d))
    q, k, v = (torch.randn(N, h, d, generator=g).bfloat16().cuda() for h in (nkv * G, nkv, nkv))
    got = []
    for p in (None, parent):
        kv, qo, out = pool.device(), torch.empty_like(q), torch.empty_like(q)
        fp.kv_append(kv, near, k, v, q=q, q_out=qo, cos=cos, sin=sin, parent=p)
        if p is None:
            fp.attn_chunk(kv, chunk, qo, out)
        else:
            fp.attn_tree(kv, chunk, p, qo, out)
        got.append([out, qo, kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else []))
    for a, b in zip(got[0][1:], got[1][1:]):
        assert torch.equal(ref.bits(a), ref.bits(b))
    # each side: its output's rounding, and probabilities rounded before they meet v (keys and values through fp16 too)
    a, b = got[0][0].double(), got[1][0].double()
    assert ((a - b).abs() <= 2 * (HALF_BF16 * b.abs() * 1.01 + (HALF_BF16 + 2.0 ** -11 + 1e-3) * v.abs().max().double())).all()


@pytest.mark.parametrize("nkv,G,d,page,kvq,lens,loose", [
    (4, 16, 128, 64, "bf16", [(8000, 64)], 0), (4, 16, 128, 64, "int8", [(8000, 64)], 0),
    (1, 8, 128, 256, "bf16", [(30001, 64), (12000, 33), (9, 64)], 0),
    (8, 8, 128, 64, "int8", [(8192, 16), (77, 16), (4000, 16)], 0),
    (2, 4, 128, 64, "int8", [(30000, 1), (10, 64), (9000, 4), (0, 0), (3, 1)], 64),
    (1, 16, 128, 32, "bf16", [(6000, 2)] * 70 + [(100, 40)], 0), (2, 2, 64, 32, "int8", [(300, 5)] * 300, 0),
])
def test_long_attention(nkv, G, d, page, kvq, lens, loose):
    """Pieces of split sequences, tiles of every size, many sequences."""
    fp = _fp()
    kv, table, g = paged._fill_gpu(lens, page, nkv, d, kvq, 31)
    chunk, starts = paged._chunk(lens, table, loose=loose)
    parent = _trees(torch.Generator().manual_seed(5), lens)
    q = torch.randn(starts[-1], nkv * G, d, generator=g, device="cuda").bfloat16()
    out = torch.empty_like(q)
    fp.attn_tree(kv, chunk, _int(parent), q, out)
    slot = ref.SLOT.cuda()
    for b, (ctx, new) in enumerate(lens):
        if new == 0 or (b > 3 and b < len(lens) - 1):
            continue
        n, r = ctx + new, starts[b]
        pos = torch.arange(n, device="cuda")
        pg, off = table[b].cuda().long()[pos // page], pos % page
        k, v = kv.k[pg, :, off].double(), kv.v[pg, :, off // 32, :, slot[off % 32]].double()
        if kvq == "int8":
            k, v = k * kv.k_scales[pg, :, off].double()[..., None], v * kv.v_scales[pg, :, off].double()[..., None]
        seen = torch.zeros(new, n, dtype=torch.bool)
        seen[:, :ctx] = True
        for i, line in enumerate(bref.lines(parent[r:r + new])):
            seen[i, ctx + torch.tensor(line)] = True
        seen = seen.cuda()
        for h in range(nkv * G):
            s = q[r:r + new, h].double() @ k[:, h // G].t().contiguous() / math.sqrt(d)
            p = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
            want, mag = p @ v[:, h // G].contiguous(), p @ v[:, h // G].abs().contiguous()
            # as in the chunk's test: scores of at most some tens keep fp32's share below 1e-4
            tol = HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * (1 + HALF_BF16)
            assert ((out[r:r + new, h].double() - want).abs() <= tol).all(), (b, h)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,loose,lens,sick", [
    (2, 4, 64, 0, [(70, 40), (0, 33), (31, 64)], [5, 7, 50]), (2, 4, 64, 32, [(70, 40), (0, 33), (31, 64)], [5, 7, 50]),
    (1, 8, 128, 0, [(70, 40), (0, 33), (31, 64)], [5, 7, 50]), (1, 8, 128, 32, [(70, 40), (0, 33), (31, 64)], [5, 7, 50]),
    (1, 8, 128, 32, [(70, 16), (0, 13), (31, 15)], [5, 7, 2]),
    (8, 8, 128, 0, [(60, 16)] * 20, [1 + b % 14 for b in range(20)]),                    # whole tiles of 128 rows, one and three
    (8, 8, 128, 0, [(290 - b, 40) for b in range(10)], [1 + 4 * b for b in range(9)] + [39]),
])
def test_values_that_are_not_finite_reach_the_nodes_that_see_them(nkv, G, d, loose, lens, sick, kvq):
    """An infinite or NaN value (and a NaN key) of one node makes its descendants' outputs what they are, and changes no
    bit of the others'."""
    fp = _fp()
    page = 32
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 25)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    parent = _trees(g, lens)
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16().cuda()
    clean, out = torch.empty_like(q), torch.empty_like(q)
    fp.attn_tree(pool.device(), chunk, _int(parent), q, clean)
    for what in ("inf", "nan", "key"):
        odd = pool.device()
        for b, node in enumerate(sick):
            pos = lens[b][0] + node
            pg, off = int(table[b, pos // page]), pos % page
            if what == "key":
                (odd.k if kvq == "bf16" else odd.k_scales)[pg, 0, off] = math.nan
            elif kvq == "bf16":
                odd.v[pg, 0, off // 32, 3, ref.SLOT[off % 32]] = math.inf if what == "inf" else math.nan
            else:
                odd.v_scales[pg, 0, off] = math.inf if what == "inf" else math.nan
        fp.attn_tree(odd, chunk, _int(parent), q, out)
        for b, (c, n) in enumerate(lens):
            see = torch.tensor([sick[b] in line for line in bref.lines(parent[starts[b]:starts[b + 1]])])
            a, w = out[starts[b]:starts[b + 1]].cpu(), clean[starts[b]:starts[b + 1]].cpu()
            assert see.any() and not see.all()
            if what == "key" or kvq == "bf16":                   # (an int8 value's scale also sets the others' rounding)
                assert torch.equal(ref.bits(a[~see]), ref.bits(w[~see]))
                assert torch.equal(ref.bits(a[see][:, G:]), ref.bits(w[see][:, G:]))
            assert torch.isfinite(a[~see].float()).all()
            bad = a[see][:, :G, 3] if kvq == "bf16" and what != "key" else a[see][:, :G]
            if what == "inf" and kvq == "bf16":
                assert (bad == math.inf).all()
            else:
                assert not torch.isfinite(bad.float()).any()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", [(2, 1, 64, 64), (3, 5, 128, 32)])
@pytest.mark.parametrize("seqs", ["edge", "ragged", "few"])
def test_append_rotates_by_depth(seqs, nkv, G, d, page, kvq):
    fp = _fp()
    lens = TREES[seqs]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 12)
    paged._fill(pool, table, lens, g)
    parent = _trees(g, lens, forest=True)
    kv = pool.device()
    chunk, starts = paged._chunk(lens, table)
    N, pad = starts[-1], 2
    cos, sin = ref.rope_tables(max(c + n for c, n in lens), d)
    q, k, v = (torch.randn(N + pad, h, d, generator=g).bfloat16() for h in (nkv * G, nkv, nkv))
    q_out = torch.full((N + pad, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    fp.kv_append(kv, chunk, k.cuda(), v.cuda(), q=q.cuda(), q_out=q_out, cos=cos.cuda(), sin=sin.cuda(), parent=_int(parent + [0] * pad))
    pos = torch.tensor(sum([[c + len(x) - 1 for x in bref.lines(parent[a:a + n])] for (c, n), a in zip(lens, starts)], []))
    qr, kr = ref.rotate(q[:N], pos, cos, sin), ref.rotate(k[:N], pos, cos, sin)
    mag = lambda x: (x[..., :d // 2].abs() + x[..., d // 2:].abs()).double().repeat(1, 1, 2)  # noqa: E731
    got = q_out.cpu()
    assert (got[N:] == 7.0).all()
    # two fp32 products and a sum, then the rounding
    assert ((got[:N].double() - qr).abs() <= HALF_BF16 * qr.abs() * (1 + 2 * EPS32) + 3 * EPS32 * mag(q[:N])).all()
    kb, vb = (torch.full((N + pad, nkv, d), 7.0, dtype=torch.bfloat16).cuda() for _ in range(2))
    fp.kv_read(kv, chunk, kb, vb)
    kb, vb = kb.cpu(), vb.cpu()
    if kvq == "bf16":
        assert ((kb[:N].double() - kr).abs() <= HALF_BF16 * kr.abs() * (1 + 2 * EPS32) + 3 * EPS32 * mag(k[:N])).all()
        assert torch.equal(vb[:N], v[:N])
    else:
        # half a code, the scale's fp16 rounding, fp32, and the bf16 read
        step = kr.abs().amax(-1, keepdim=True) / 127
        assert ((kb[:N].double() - kr).abs() <= step * (0.5 + 127 * 2.0 ** -11) * 1.01 + HALF_BF16 * kr.abs() * 1.01).all()
        c, s = ref.quantise(v[:N].float())
        assert torch.equal(vb[:N], (c.float() * s.float()[..., None]).bfloat16())
    # without angles the parents do not matter
    a, b = pool.device(), pool.device()
    fp.kv_append(a, chunk, k.cuda(), v.cuda())
    fp.kv_append(b, chunk, k.cuda(), v.cuda(), parent=_int(parent + [0] * pad))
    assert torch.equal(ref.bits(a.k), ref.bits(b.k)) and torch.equal(ref.bits(a.v), ref.bits(b.v))


# ------------------------------------------------------------------ the accepted path
def _moved(pool, table, lens, path, keep, R):
    """The pool after the move, bit for bit: tensors of the cache."""
    new = [t.clone() for t in pool.tensors()]
    for b, (c, n) in enumerate(lens):
        for j in range(max(0, min(keep[b], R, n))):
            s = path[b][j]
            if not 0 <= s < n:
                continue
            (pa, oa), (pt, ot) = (pool._at(table[b], torch.tensor([c + x])) for x in (s, j))
            if not 0 <= int(pt) < pool.n_pages:
                continue
            ok = 0 <= int(pa) < pool.n_pages
            pa = pa if ok else torch.zeros_like(pa)
            new[0][pt, :, ot] = pool.k[pa, :, oa] if ok else torch.zeros_like(pool.k[pa, :, oa])
            v = pool.v[pa, :, oa // 32, :, ref.SLOT[oa % 32]]
            new[1][pt, :, ot // 32, :, ref.SLOT[ot % 32]] = v if ok else torch.zeros_like(v)
            for i, t in ((2, pool.ks), (3, pool.vs)):
                if t is not None:
                    new[i][pt, :, ot] = t[pa, :, oa] if ok else torch.zeros_like(t[pa, :, oa])
    return new


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,d,page", [(1, 64, 32), (3, 128, 96), (8, 64, 64)])
def test_keep_moves_any_path(nkv, d, page, kvq):
    """Paths in order and not, with gaps and repeats, entries and counts out of range, a missing page; the rest of the pool
    stays bit for bit."""
    fp = _fp()
    lens = [(30, 64), (0, 5), (64, 0), (95, 33), (17, 8), (200, 64), (31, 1), (10, 40)]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 33)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    R = 50
    path = [[int(x) for x in torch.randint(-1, 70, (R,), generator=g)] for _ in lens]
    path[0] = list(range(14, 64))                               # each overwrites what a later one reads
    path[3] = [0, 2, 3, 7, 20, 21, 32] + [-1] * (R - 7)
    path[5] = list(range(63, 13, -1))
    path[1][:6] = [4, 3, 2, 1, 0, 2**31 - 1]
    keep = [64, 6, 3, 7, -4, 2**31 - 1, 1, 20]
    table[7, (10 + 5) // page if page == 32 else 0] = -9
    kvs = [pool.device() for _ in range(3)]
    chunk, _ = paged._chunk(lens, table, max_new=64)
    fp.kv_keep(kvs, chunk, _int(path), _int(keep))
    want = _moved(pool, table, lens, path, keep, R)
    for kv in kvs:
        for a, w in zip([kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else []), want):
            assert torch.equal(ref.bits(a.cpu()), ref.bits(w))
    one = pool.device()
    fp.kv_keep(one, chunk, _int(path), _int(keep))
    assert torch.equal(ref.bits(one.k.cpu()), ref.bits(want[0]))


def test_keep_in_many_layers_of_both_formats():
    fp = _fp()
    lens, page, nkv, d = [(40, 9), (3, 30)], 32, 2, 64
    pools, tabs = [], None
    for i in range(70):
        g, pool, table = paged._case(lens, page, nkv, d, "int8" if 34 <= i < 36 or i % 7 == 6 else "bf16", 35)
        paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
        pools.append(pool)
        tabs = table
    kvs = [p.device() for p in pools]
    path, keep = [[0, 3, 8, -1], [0, 1, 7, 29]], [3, 4]
    chunk, _ = paged._chunk(lens, tabs)
    fp.kv_keep(kvs, chunk, _int(path), _int(keep))
    for kv, pool in zip(kvs, pools):
        want = _moved(pool, tabs, lens, path, keep, 4)
        for a, w in zip([kv.k, kv.v, kv.k_scales, kv.v_scales], want):
            assert torch.equal(ref.bits(a.cpu()), ref.bits(w))


# ------------------------------------------------------------------ verification
def _verify(logits, starts, parent, ids, u, T, R, stride=None):
    fp = _fp()
    N, V = logits.shape
    B = len(starts) - 1
    z = logits.cuda()
    if stride is not None:                                       # rows of a wider buffer, off 16-byte steps
        w = torch.full((N, V + stride), math.nan).cuda()
        w[:, 1:V + 1] = z
        z = w[:, 1:V + 1]
    out, path = (torch.full((B, R), 77, dtype=torch.int32).cuda() for _ in range(2))
    n = torch.full((B,), 77, dtype=torch.int32).cuda()
    fp.verify_tree(z, _int(starts), _int(parent), _int(ids), u.cuda() if u is not None else None, out, path, n, temperature=T)
    want = bref.verify_tree(logits, starts, parent, ids, u, T, R)
    assert n.cpu().tolist() == [len(t) for t, _ in want]
    pad = lambda x: x + [-1] * (R - len(x))  # noqa: E731
    assert out.cpu().tolist() == [pad(t) for t, _ in want]
    assert path.cpu().tolist() == [pad(p) for _, p in want]
    return want


def _likely(g, logits, starts, parent, T):
    """Tokens of the nodes: mostly likely ones after their parents."""
    ids = torch.randint(logits.shape[1], (logits.shape[0],), generator=g).tolist()
    for a, b in zip(starts, starts[1:]):
        for i in range(1, b - a):
            p = parent[a + i]
            if 0 <= p < i:
                e = -torch.log(-torch.log(torch.rand(logits.shape[1], generator=g)))
                ids[a + i] = int((logits[a + p] + max(T, 0.2) * e).argmax())
    return ids


@pytest.mark.parametrize("T", [0.0, 0.3, 1.0, 2.5])
@pytest.mark.parametrize("rows,V", [([1], 1), ([7], 17), ([20, 1, 33, 3], 1000), ([16] * 9, 4096), ([30, 0, 20], 4097),
                                    ([64, 1, 20], 333), ([9, 5], 33001)])
def test_paths_match(rows, V, T):
    g = torch.Generator().manual_seed(len(rows) + V)
    starts = np.cumsum([0] + rows).tolist()
    # rows peaked enough that drafted tokens are drawn
    logits = 2 * torch.randn(starts[-1], V, generator=g)
    logits.scatter_add_(1, torch.randint(V, (starts[-1], 3), generator=g), 8 * torch.rand(starts[-1], 3, generator=g))
    parent = sum([bref.random_tree(g, n, forest=V == 1000) for n in rows if n], [])
    for rep in range(3):
        ids, u = _likely(g, logits, starts, parent, T), torch.rand(starts[-1], generator=g)
        _verify(logits, starts, parent, ids, u if T > 0 else None, T, max(rows), stride=3 if rep else None)


@pytest.mark.parametrize("T", [0.0, 1.0])
def test_verification_of_odd_rows(T):
    """Equal logits, infinities, NaN, rows without any probability, duplicate children, more rows than max_rows, drafts
    that are no tokens, u of zero and of almost one."""
    g = torch.Generator().manual_seed(3)
    V, n = 5000, 24
    logits = torch.randn(2 * n, V, generator=g)
    logits[0] = 0.0                                              # all equal
    logits[1, [7, 4900]] = math.inf
    logits[2] = math.nan
    logits[3] = -math.inf
    logits[4, ::3] = math.nan
    logits[5] = torch.finfo(torch.float32).min
    logits[5, 4999] = 3.0
    logits[n:] = logits[:n]
    parent = [-1] + [0] * 8 + [int(torch.randint(0, 9, (1,), generator=g)) for _ in range(n - 9)]
    parent = parent + parent
    starts = [0, n, 2 * n]
    for u0 in (0.0, 0.3, 1.0 - 2.0 ** -24):
        u = torch.full((2 * n,), u0)
        # children of the root hold what it draws, in turn
        first = _verify(logits, starts, parent, [-1] * (2 * n), u, T, n)
        y = first[0][0][0]
        for child in range(1, 9):
            ids = [-1] * (2 * n)
            for c in (child, 8):                                 # a duplicate: the first counts
                ids[c] = ids[n + c] = y
            second = _verify(logits, starts, parent, ids, u, T, n)
            assert second[0][1][:2] == [0, child]
            z = second[0][0][1]
            for j in range(9, n):
                if parent[j] == child:
                    ids[j] = ids[n + j] = z                      # -1 where the child has no probability: never accepted
            _verify(logits, starts, parent, ids, u, T, n)
    # more rows than max_rows: cut
    _verify(logits, [0, 2 * n], parent, [-1] * (2 * n), torch.full((2 * n,), 0.5), T, 5)


def test_verification_over_the_largest_vocabulary():
    g = torch.Generator().manual_seed(4)
    V = 1 << 20
    logits = torch.randn(3, V, generator=g)
    for T in (0.0, 1.0):
        for u in (0.0, 0.77, 1.0 - 2.0 ** -24):
            first = _verify(logits, [0, 3], [-1, 0, 1], [0, 0, 0], torch.full((3,), u), T, 3)
            _verify(logits, [0, 3], [-1, 0, 1], [0, first[0][0][0], 5], torch.full((3,), u), T, 3)


# ------------------------------------------------------------------ the layer stack, and a run of it all
EXTEND = [("bf16", "bf16", Shape(2, 256, 4, 4, 64, 688, 4, 64, 200), 32), ("int8", "int8", Shape(2, 512, 8, 2, 64, 768, 3, 96, 160), 64),
          ("int4", "bf16", Shape(1, 640, 5, 1, 128, 768, 64, 40, 150), 96), ("sp24", "int8", Shape(1, 256, 4, 2, 64, 448, 2, 128, 140), 32)]


@pytest.mark.parametrize("wq,kvq,s,page", EXTEND)
def test_extended_trees_are_their_lines(wq, kvq, s, page):
    """Every node's output is that of the oracle for the sequence from the first token along the node's line."""
    import paper_2501_13111_amd as fp
    from oracle.layer import Fingerprint as OracleFingerprint
    from oracle.numerics import bf16_round
    rng, g = np.random.default_rng(13), torch.Generator().manual_seed(13)
    ctx, nodes = [20, 0, 33], [13, 7, 1]
    prompt = [bf16_round(rng.normal(0, 1, (c, s.hidden)).astype(np.float32)) for c in ctx]
    tree = [bf16_round(rng.normal(0, 1, (n, s.hidden)).astype(np.float32)) for n in nodes]
    parent = [bref.random_tree(g, n) for n in nodes]
    orc = OracleFingerprint(s, wq, kvq, seed=4)
    with fp.Fingerprint(s, wq, kvq, seed=4) as f:
        p = Paged(f, kvq, page, [60] * 3)
        p.extend(prompt)
        starts = np.cumsum([0] + nodes).tolist()
        chunk = fp.Chunk(_int(starts), _int(ctx), p.table, max_new=max(nodes), max_len=60)
        x = np_to_bf16(np.concatenate(tree))
        y = torch.empty_like(x)
        f.extend(p.kvs, chunk, x, y, parent=_int(sum(parent, [])))
        got = bf16_to_np(y)
    errs = []
    for b in range(3):
        for i, line in enumerate(bref.lines(parent[b])):
            want = orc.prefill(np.concatenate([prompt[b], tree[b][line]])[None])[0]
            errs.append(rel_inf(got[starts[b] + i][None], want[-1:]))
    assert max(errs) <= TOL, errs


@pytest.mark.parametrize("T", [0.0, 0.8])
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
def test_tree_decoding_run(kvq, T):
    """Embedding, layers over trees, LM head of every node, decision, the accepted path kept, and on: the tokens are the
    reference's decision on those logits, and the logits of every root are what a fingerprint that was fed the
    accepted tokens one by one gives."""
    import paper_2501_13111_amd as fp
    s = Shape(2, 256, 4, 2, 64, 448, 32, 16, 96, vocab=512)
    B, n = 3, 9
    g = torch.Generator().manual_seed(9)
    with fp.Fingerprint(s, "bf16", kvq, seed=10) as f:
        trees, plain = Paged(f, kvq, 32, [90] * B), Paged(f, kvq, 64, [90] * B, seed=1)
        hist = [torch.randint(s.vocab, (m,), generator=g).tolist() for m in (7, 12, 31)]

        def layers(p, toks, parent=None):
            ids = _int(sum(toks, []))
            x = torch.empty(len(ids), s.hidden, dtype=torch.bfloat16, device="cuda")
            f.embed(ids, x)
            starts = np.cumsum([0] + [len(t) for t in toks]).tolist()
            chunk = fp.Chunk(_int(starts), _int(p.pos), p.table, max_new=max(len(t) for t in toks), max_len=90)
            y, lg = torch.empty_like(x), torch.empty(len(ids), s.vocab, device="cuda")
            f.extend(p.kvs, chunk, x, y, parent=None if parent is None else _int(parent))
            nxt = torch.empty(len(ids), dtype=torch.int32, device="cuda")
            for a in range(0, len(ids), s.max_batch):
                b = min(a + s.max_batch, len(ids))
                f.head(y[a:b], b - a, 1, nxt[a:b], lg[a:b])
            return chunk, starts, lg

        for p in (trees, plain):
            layers(p, [h[:-1] for h in hist])
            p.pos = [len(h) - 1 for h in hist]
        accepted = 0
        for it in range(5):
            parent = sum([bref.random_tree(g, n) for _ in range(B)], [])
            toks = [[h[-1]] + torch.randint(s.vocab, (n - 1,), generator=g).tolist() for h in hist]
            # what the plain fingerprint would say after the root, at two of the root's children
            _, _, lg = layers(plain, [[h[-1]] for h in hist])
            for b in range(B):
                kids = [i for i in range(1, n) if parent[b * n + i] == 0]
                toks[b][kids[-1]] = int(lg[b].argmax())
            chunk, starts, lt = layers(trees, toks, parent)
            assert rel_inf(lt[starts[:-1]].cpu().numpy(), lg.cpu().numpy()) <= TOL
            u = torch.rand(B * n, generator=g)
            out, path = (torch.empty(B, n, dtype=torch.int32, device="cuda") for _ in range(2))
            count = torch.empty(B, dtype=torch.int32, device="cuda")
            fp.verify_tree(lt, _int(starts), _int(parent), _int(sum(toks, [])), u.cuda(), out, path, count, temperature=T)
            want = bref.verify_tree(lt.cpu(), starts, parent, sum(toks, []), u, T, n)
            assert [(out[b, :count[b]].tolist(), path[b, :count[b]].tolist()) for b in range(B)] == want
            fp.kv_keep(trees.kvs, chunk, path, count)
            # the plain one takes the accepted tokens (the root is in already)
            plain.pos = [x + 1 for x in plain.pos]
            rest = [t[:-1] for t, _ in want]
            if any(rest):
                layers(plain, rest)
            for b in range(B):
                plain.pos[b] += len(rest[b])
                trees.pos[b] += len(want[b][0])
                hist[b] += want[b][0]
                accepted += len(rest[b])
            assert trees.pos == plain.pos
    assert accepted > 0 or T > 0        # (at T the nearly flat logits accept one token in hundreds)


def test_captured_trees_follow_their_contents():
    """Append, attention, verification and the move in one graph, replayed with other lengths, trees and tokens, with eager work of
    the same calls between the replays; two graphs with a workspace each, side by side."""
    fp = _fp()
    nkv, G, d, page, B, n, V, L = 2, 4, 64, 32, 3, 10, 700, 2
    g = torch.Generator().manual_seed(51)
    cos, sin = (t.cuda() for t in ref.rope_tables(300, d))

    class Side:
        def __init__(self):
            self.kvs = []
            for _ in range(L):
                gg, pool, table = paged._case([(280, n)] * B, page, nkv, d, "int8", 52)
                paged._fill(pool, table, [(280, n)] * B, gg, upto=lambda c, m: c + m)
                self.kvs.append(pool.device())
            self.row_start, self.ctx = _int([0] * (B + 1)), _int([0] * B)
            self.chunk = fp.Chunk(self.row_start, self.ctx, table.cuda(), max_new=n, max_len=290)
            N = B * n
            self.parent, self.ids = _int([-1] * N), _int([0] * N)
            self.q, self.qr, self.out = (torch.zeros(N, nkv * G, d, dtype=torch.bfloat16).cuda() for _ in range(3))
            self.k, self.v = (torch.zeros(N, nkv, d, dtype=torch.bfloat16).cuda() for _ in range(2))
            self.lg, self.u = torch.zeros(N, V).cuda(), torch.zeros(N).cuda()
            self.toks, self.path, self.count = _int([[0] * n] * B), _int([[0] * n] * B), _int([0] * B)
            self.ws = fp.attn_chunk_workspace(self.kvs[0], self.chunk, N, nkv * G)
            self.vws = fp.verify_tree_workspace(N, V)

        def run(self):
            for kv in self.kvs:
                fp.kv_append(kv, self.chunk, self.k, self.v, q=self.q, q_out=self.qr, cos=cos, sin=sin, parent=self.parent)
                fp.attn_tree(kv, self.chunk, self.parent, self.qr, self.out, workspace=self.ws)
            fp.verify_tree(self.lg, self.row_start, self.parent, self.ids, self.u, self.toks, self.path, self.count, temperature=0.7,
                           workspace=self.vws)
            fp.kv_keep(self.kvs, self.chunk, self.path, self.count)

        def state(self):
            return [self.out, self.qr, self.toks, self.path, self.count] + [t for kv in self.kvs for t in (kv.k, kv.v, kv.k_scales, kv.v_scales)]

    sides = [Side() for _ in range(3)]                           # two captured, one eager
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs = []
    for s in sides[:2]:
        s.run()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            s.run()
        graphs.append(gr)
    sides[2].run()
    for it in range(6):
        rows = [[10, 3, 7], [1, 10, 0], [4, 4, 4], [10, 10, 10], [2, 9, 1], [5, 0, 8]][it]
        starts = np.cumsum([0] + rows).tolist()
        ctx = [[0, 31, 270], [280, 5, 64], [90, 63, 33], [200, 12, 100], [150, 96, 1], [0, 0, 95]][it]
        parent = sum([bref.random_tree(g, m) for m in rows if m], [])
        N = len(parent)
        data = {"q": torch.randn(N, nkv * G, d, generator=g).bfloat16(), "k": torch.randn(N, nkv, d, generator=g).bfloat16(),
                "v": torch.randn(N, nkv, d, generator=g).bfloat16(), "lg": 4 * torch.randn(N, V, generator=g), "u": torch.rand(N, generator=g),
                "parent": torch.tensor(parent, dtype=torch.int32)}
        data["ids"] = torch.tensor(_likely(g, data["lg"], starts, parent, 0.7), dtype=torch.int32)
        for s in sides:
            s.row_start.copy_(_int(starts))
            s.ctx.copy_(_int(ctx))
            for name, t in data.items():
                getattr(s, name)[:N].copy_(t.cuda())
        torch.cuda.synchronize()
        sides[2].run()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for s in sides[:2]:
            for a, b in zip(s.state(), sides[2].state()):
                assert torch.equal(ref.bits(a), ref.bits(b)), it


def test_trees_on_another_stream():
    """On a stream of the caller's, with workspaces of its own; without them another stream is refused."""
    fp = _fp()
    lens, page, nkv, G, d = [(100, 12), (40, 20)], 32, 2, 2, 64
    g, pool, table = paged._case(lens, page, nkv, d, "bf16", 61)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    parent = _trees(g, lens)
    chunk, starts = paged._chunk(lens, table)
    N = starts[-1]
    kv, q = pool.device(), torch.randn(N, nkv * G, d, generator=g).bfloat16().cuda()
    want, out = torch.empty_like(q), torch.empty_like(q)
    pp = _int(parent)
    fp.attn_tree(kv, chunk, pp, q, want)
    st = torch.cuda.Stream()
    ws = fp.attn_chunk_workspace(kv, chunk, N, nkv * G)
    torch.cuda.synchronize()
    fp.attn_tree(kv, chunk, pp, q, out, workspace=ws, stream=st)
    st.synchronize()
    assert torch.equal(out, want)
    with pytest.raises(ValueError, match="workspace"):
        fp.attn_tree(kv, chunk, pp, q, out, stream=st)
    with pytest.raises(ValueError, match="parent"):
        fp.attn_tree(kv, chunk, pp[:-1], q, out)
    with pytest.raises(ValueError, match="parent"):
        fp.attn_tree(kv, chunk, pp.long(), q, out)
    lg, ids = torch.randn(N, 50).cuda(), _int([0] * N)
    o, h, n = torch.empty(2, 20, dtype=torch.int32).cuda(), torch.empty(2, 20, dtype=torch.int32).cuda(), _int([0, 0])
    with pytest.raises(ValueError, match="workspace"):
        fp.verify_tree(lg, chunk.row_start, pp, ids, None, o, h, n, temperature=0, stream=st)
    with pytest.raises(ValueError, match="path"):
        fp.verify_tree(lg, chunk.row_start, pp, ids, None, o, h[:, 1:], n, temperature=0)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
def test_pages_past_32_bits_of_bytes(kvq):
    """Append, attention (16 nodes: streamed, in tiles of 64 or 32, and of 128), the move and the beams' copies among the last pages of
    a pool above 4 GiB leave the same bits as in a small pool."""
    fp = _fp()
    lens, page, nkv, d = [(700, 16), (300, 12), (0, 16), (1000, 7)], 256, 8, 128
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 71)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    parent = _int(_trees(g, lens))
    N = sum(n for _, n in lens)
    small = pool.device()
    n = small.n_pages
    big = fp.PagedKV.empty((9 << 29) // (nkv * page * d * small.k.element_size()), page, nkv, d, kvq)
    assert big.k.nbytes > 1 << 32
    hi = big.n_pages - n

    def held(kv, at):
        ts = [kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else [])
        return [t[at:at + n] for t in ts]

    for a, b in zip(held(small, 0), held(big, hi)):
        b.copy_(a)
    cos, sin = torch.rand(2, 1100, d // 2, generator=g).cuda()
    k, v = torch.randn(2, N, nkv, d, generator=g).bfloat16().cuda()
    out = []
    for kv, at in ((small, 0), (big, hi)):
        tab = torch.where((table >= 0) & (table < n), table + at, -1).int()
        res = []
        for G in (1, 2, 8):
            q = torch.randn(N, nkv * G, d, generator=torch.Generator().manual_seed(G)).bfloat16().cuda()
            qr = torch.empty_like(q)
            fp.kv_append(kv, paged._chunk(lens, tab)[0], k, v, q=q, q_out=qr, cos=cos, sin=sin, parent=parent)
            res.append(qr)
            for loose in (0, page):
                o = torch.empty_like(q)
                fp.attn_tree(kv, paged._chunk(lens, tab, loose=loose)[0], parent, qr, o)
                res.append(o)
        fp.kv_keep(kv, paged._chunk(lens, tab)[0], _int([[0, 3, 5, 6]] * 4), _int([4, 3, 2, 4]))
        tab = tab.cuda()
        fp.beam_reorder(kv, tab, _int([700] * 4), _int([[1, 1, 0, 1]]))
        out.append(res + held(kv, at) + [torch.where(tab >= 0, tab - at, -1).int()])
    for a, b in zip(*out):
        assert torch.equal(ref.bits(a.cpu()), ref.bits(b.cpu()))
