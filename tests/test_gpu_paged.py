"""The paged cache on the GPU against a plain 64-bit reference: writing a chunk (rotation, int8
quantisation), reading back, and attention of a chunk over the pages."""
import math

import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu

HALF_BF16 = 2.0 ** -8        # largest relative error of a rounding to bf16
EPS32 = 2.0 ** -24


def _fp():
    import paper_2501_13111_amd as fp
    return fp


def _case(lens, page, nkv, d, kvq, seed, width=None, spare=2):
    """CPU pool and table for sequences of lens = [(ctx, new)]."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-(c + n) // page) for c, n in lens]
    n_pages = sum(need) + spare
    width = width or max(max(need), 1) + 1
    pool = ref.Pool(n_pages, page, nkv, d, kvq)
    return g, pool, ref.tables(g, need, n_pages, width)


def _fill(pool, table, lens, g, upto=lambda c, n: c, scale=1.0):
    for b, (c, n) in enumerate(lens):
        m = upto(c, n)
        if m:
            pool.write(table[b], torch.arange(m), scale * torch.randn(m, pool.nkv, pool.d, generator=g).bfloat16().float(),
                       torch.randn(m, pool.nkv, pool.d, generator=g).bfloat16().float())


def _chunk(lens, table, extra_rows=0, max_len=None, max_new=None, loose=0):
    """loose: a bound on the positions far beyond the sequences' (pages of this size), which large calls have:
    more than 64 rows to a kv head then take the kernel of 256-row tiles."""
    fp = _fp()
    if loose:
        max_len = 1 << 22
        table = torch.nn.functional.pad(table, (0, max_len // loose + 1 - table.shape[1]), value=-7)
    starts = [0]
    for _, n in lens:
        starts.append(starts[-1] + n)
    c = fp.Chunk(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor([c for c, _ in lens], dtype=torch.int32).cuda(),
                 table.cuda(), max_new=max_new or max(1, max(n for _, n in lens)),
                 max_len=max_len or max(1, max(c + n for c, n in lens)))
    return c, starts


SEQS = {
    "one": [(0, 1)],
    "token": [(331, 1)],
    "edge": [(31, 1), (32, 1), (63, 2), (0, 32), (0, 33), (95, 1)],
    "ragged": [(5, 3), (0, 0), (100, 1), (64, 0), (33, 70), (0, 1)],
    "empty-first": [(7, 0), (0, 0), (40, 9)],
    "chunk": [(130, 161)],
}


# ------------------------------------------------------------------ append and read
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", [(1, 1, 64, 32), (3, 5, 128, 96), (8, 2, 64, 128)])
@pytest.mark.parametrize("seqs", sorted(SEQS))
def test_append_matches_the_reference_bit_for_bit(seqs, nkv, G, d, page, kvq):
    """Keys that arrive rotated: codes, scales and every untouched byte of the pool."""
    fp = _fp()
    lens = SEQS[seqs]
    g, pool, table = _case(lens, page, nkv, d, kvq, 11)
    _fill(pool, table, lens, g)
    kv = pool.device()
    chunk, starts = _chunk(lens, table)
    N = starts[-1]
    fused = torch.randn(N + 3, (G + 2) * nkv, d, generator=g).bfloat16()
    fused[:, :, 5] *= 100                                       # an outlier channel
    if N > 1:
        fused[1] = 0                                            # a zero row: zero scale, zero codes
    k, v = fused[:, G * nkv:(G + 1) * nkv], fused[:, (G + 1) * nkv:]
    dev = fused.cuda()
    fp.kv_append(kv, chunk, dev[:, G * nkv:(G + 1) * nkv], dev[:, (G + 1) * nkv:])
    for b, (c, n) in enumerate(lens):
        if n:
            pool.write(table[b], torch.arange(c, c + n), k[starts[b]:starts[b + 1]].float(), v[starts[b]:starts[b + 1]].float())
    got = [kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else [])
    for a, want in zip(got, pool.tensors()):
        assert torch.equal(ref.bits(a.cpu()), ref.bits(want))


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", [(2, 1, 64, 64), (3, 5, 128, 32), (2, 16, 128, 96)])
@pytest.mark.parametrize("seqs", ["edge", "ragged", "chunk"])
def test_append_rotates(seqs, nkv, G, d, page, kvq):
    fp = _fp()
    lens = SEQS[seqs]
    g, pool, table = _case(lens, page, nkv, d, kvq, 12)
    _fill(pool, table, lens, g)
    kv = pool.device()
    chunk, starts = _chunk(lens, table)
    N, pad = starts[-1], 2
    cos, sin = ref.rope_tables(max(c + n for c, n in lens) + 3, d)
    q, k, v = (torch.randn(N + pad, h, d, generator=g).bfloat16() for h in (nkv * G, nkv, nkv))
    q_out = torch.full((N + pad, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    fp.kv_append(kv, chunk, k.cuda(), v.cuda(), q=q.cuda(), q_out=q_out, cos=cos.cuda(), sin=sin.cuda())
    pos = torch.cat([torch.arange(c, c + n) for c, n in lens])
    # fp32 rotation: two products and a sum, each off by at most EPS32 of |x c| + |y s|
    qr, kr = ref.rotate(q[:N], pos, cos, sin), ref.rotate(k[:N], pos, cos, sin)
    mag = lambda x: (x[..., :d // 2].abs() + x[..., d // 2:].abs()).double().repeat(1, 1, 2)  # noqa: E731
    got = q_out.cpu()
    assert (got[N:] == 7.0).all()                               # rows behind the last sequence
    assert ((got[:N].double() - qr).abs() <= HALF_BF16 * qr.abs() * (1 + 2 * EPS32) + 3 * EPS32 * mag(q[:N])).all()
    kb, vb = (torch.full((N + pad, nkv, d), 7.0, dtype=torch.bfloat16).cuda() for _ in range(2))
    fp.kv_read(kv, chunk, kb, vb)
    kb, vb = kb.cpu(), vb.cpu()
    assert (kb[N:] == 7.0).all() and (vb[N:] == 7.0).all()
    if kvq == "bf16":
        assert ((kb[:N].double() - kr).abs() <= HALF_BF16 * kr.abs() * (1 + 2 * EPS32) + 3 * EPS32 * mag(k[:N])).all()
        assert torch.equal(vb[:N], v[:N])
    else:
        # half a code, the scale's fp16 rounding (2^-11 of at most 127 codes), fp32, and the bf16 read
        step = kr.abs().amax(-1, keepdim=True) / 127
        tol = step * (0.5 + 127 * 2.0 ** -11) * 1.01 + HALF_BF16 * kr.abs() * 1.01
        assert ((kb[:N].double() - kr).abs() <= tol).all()
        c, s = ref.quantise(v[:N].float())
        assert torch.equal(vb[:N], (c.float() * s.float()[..., None]).bfloat16())


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,d,page,lens", [(1, 64, 32, [(0, 1)]), (5, 128, 160, [(0, 333), (0, 0), (0, 32), (0, 31)]),
                                             (4, 64, 64, [(17, 50), (64, 64), (3, 1)])])
def test_read_returns_what_the_pages_hold(nkv, d, page, lens, kvq):
    fp = _fp()
    g, pool, table = _case(lens, page, nkv, d, kvq, 13)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n)
    chunk, starts = _chunk(lens, table)
    N = starts[-1]
    k, v = (torch.full((N + 2, nkv, d), 7.0, dtype=torch.bfloat16).cuda() for _ in range(2))
    fp.kv_read(pool.device(), chunk, k, v)
    for b, (c, n) in enumerate(lens):
        if n:
            wk, wv = pool.read(table[b], c + n)
            # codes times an fp16 scale are exact in fp32, so one rounding to bf16
            assert torch.equal(k[starts[b]:starts[b + 1]].cpu(), wk[c:].float().bfloat16())
            assert torch.equal(v[starts[b]:starts[b + 1]].cpu(), wv[c:].float().bfloat16())
    assert (k[N:] == 7.0).all() and (v[N:] == 7.0).all()


# ------------------------------------------------------------------ attention
def _check_attention(pool, table, lens, q, out, scale=None, fp16=False, floor=0.0):
    """fp16: int8 keys and values that meet the matrix cores as fp16 (half a step is 2^-11)."""
    want, mag, smag = ref.attention(pool, table, lens, q, scale)
    N = want.shape[0]
    d = q.shape[2]
    # output rounding; probabilities rounded to bf16 before they meet v (their sum is not); fp32
    # scores of d products, each side of the quotient off by the largest score error
    ds = 2 * (d + 4) * EPS32 * smag
    if fp16:
        ds = ds + 2 * 2.0 ** -11 * smag
    tol = HALF_BF16 * want.abs() + (HALF_BF16 + 2 * ds + 1e-5 + (2.0 ** -11 if fp16 else 0.0)) * mag * (1 + HALF_BF16) + floor
    err = (out[:N].cpu().double() - want).abs()
    assert (err <= tol).all(), f"{(err / tol.clamp(min=1e-30)).max():.3f} of the tolerance"


SHAPES = [(1, 1, 64, 32), (2, 4, 128, 64), (3, 5, 128, 96), (2, 16, 64, 32), (4, 3, 64, 128), (1, 8, 128, 256)]
ATTN_SEQS = dict(SEQS, **{
    "drafts": [(200, 5), (31, 5), (0, 5), (511, 2)],
    "long": [(2500, 1), (3, 1), (1100, 1)],
    "split-drafts": [(1700, 4), (90, 6)],
    "far-chunk": [(2300, 40), (17, 90)],
    "mixed": [(40, 1), (250, 130), (700, 1), (0, 200)],
})


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", SHAPES)
@pytest.mark.parametrize("seqs", sorted(ATTN_SEQS))
def test_attention_matches_the_reference(seqs, nkv, G, d, page, kvq, loose):
    fp = _fp()
    lens = ATTN_SEQS[seqs]
    g, pool, table = _case(lens, page, nkv, d, kvq, 21)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n, scale=1.5)
    kv = pool.device()
    chunk, starts = _chunk(lens, table, loose=page * loose)
    N = starts[-1]
    q = torch.randn(N + 2, nkv * G, d, generator=g).bfloat16()
    out = torch.full((N + 2, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    fp.attn_chunk(kv, chunk, q.cuda(), out)
    assert (out[N:] == 7.0).all()
    _check_attention(pool, table, lens, q[:N], out)
    again = torch.empty_like(out)
    fp.attn_chunk(kv, chunk, q.cuda(), again)
    assert torch.equal(ref.bits(again[:N]), ref.bits(out[:N]))


def _gpu_attention(kv, table, lens, q):
    """The reference in 64 bits on the device, for lengths that loops would not finish."""
    d, nkv, H = kv.head_dim, kv.n_kv_heads, q.shape[1]
    G, slot = H // nkv, ref.SLOT.cuda()
    out, mag, r = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda"), 0
    for b, (ctx, new) in enumerate(lens):
        n = ctx + new
        pos = torch.arange(n, device="cuda")
        pg, off = table[b].cuda().long()[pos // kv.page_size], pos % kv.page_size
        k, v = kv.k[pg, :, off].double(), kv.v[pg, :, off // 32, :, slot[off % 32]].double()
        if kv.kvq == "int8":
            k, v = k * kv.k_scales[pg, :, off].double()[..., None], v * kv.v_scales[pg, :, off].double()[..., None]
        for h in range(H):
            s = q[r:r + new, h].double() @ k[:, h // G].t().contiguous() / math.sqrt(d)
            s.masked_fill_(pos[None, :] > ctx + torch.arange(new, device="cuda")[:, None], -math.inf)
            p = torch.softmax(s, -1)
            out[r:r + new, h] = p @ v[:, h // G].contiguous()
            mag[r:r + new, h] = p @ v[:, h // G].abs().contiguous()
        r += new
    return out, mag


def _fill_gpu(lens, page, nkv, d, kvq, seed, spare=2):
    """A pool on the device with every position of the sequences written by kv_append."""
    fp = _fp()
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-(c + n) // page) for c, n in lens]
    table = ref.tables(torch.Generator().manual_seed(seed), need, sum(need) + spare, max(need))
    kv = fp.PagedKV.empty(sum(need) + spare, page, nkv, d, kvq)
    whole, starts = _chunk([(0, c + n) for c, n in lens], table)
    k = (1.5 * torch.randn(starts[-1], nkv, d, generator=g, device="cuda")).bfloat16()
    v = torch.randn(starts[-1], nkv, d, generator=g, device="cuda").bfloat16()
    fp.kv_append(kv, whole, k, v)
    return kv, table, g


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("nkv,G,d,page,kvq,lens", [
    (4, 16, 128, 64, "bf16", [(8000, 130)]),          # pieces of more than 64 blocks, many tiles
    (4, 16, 128, 64, "int8", [(8000, 130)]),
    (2, 1, 64, 32, "int8", [(5000, 700), (9, 1000)]),
    (8, 2, 128, 256, "bf16", [(0, 1000), (0, 3), (0, 517)]),
    (1, 8, 128, 128, "int8", [(70000, 1), (33, 1), (40000, 1)]),
    (8, 1, 64, 96, "bf16", [(20000, 2)] * 3),
    # next tokens and a few rows beside chunks
    (2, 4, 128, 64, "int8", [(30000, 1), (10, 100), (9000, 4), (0, 0), (3, 1)]),
    (2, 4, 64, 64, "bf16", [(40, 1), (20000, 2), (3000, 300), (7000, 1), (5, 5), (8000, 4), (0, 70)]),
    (1, 16, 128, 32, "bf16", [(6000, 1)] * 70 + [(100, 40)]),
    (3, 1, 64, 32, "int8", [(9000, 16), (9000, 17), (50, 70)]),
])
def test_long_attention(nkv, G, d, page, kvq, lens, loose):
    fp = _fp()
    kv, table, g = _fill_gpu(lens, page, nkv, d, kvq, 31)
    chunk, starts = _chunk(lens, table, loose=page * loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g, device="cuda").bfloat16()
    out = torch.empty_like(q)
    fp.attn_chunk(kv, chunk, q, out)
    want, mag = _gpu_attention(kv, table, lens, q)
    # as in _check_attention; scores of at most some tens keep fp32's share below 1e-4
    assert ((out.double() - want).abs() <= HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * (1 + HALF_BF16)).all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,new,loose", [(2, 2, 1, 0), (1, 8, 5, 0), (2, 4, 90, 0), (2, 4, 90, 64)])
def test_scores_far_apart_and_rising(nkv, G, new, loose, kvq):
    """Keys whose scores grow along the sequence (the softmax's reference moves again and again), tiny and
    large values beside each other, a negative scale, q at the top of bf16's useful range."""
    fp = _fp()
    d, page, lens = 128, 64, [(900, new), (333, new)]
    for scale, qs in ((None, 1.0), (-0.05, 1.0), (1e-7, 3e5), (3.0, 0.2)):
        g, pool, table = _case(lens, page, nkv, d, kvq, 41)
        for b, (c, n) in enumerate(lens):
            m = c + n
            ramp = torch.linspace(0.1, 6, m)[:, None, None]
            pool.write(table[b], torch.arange(m), (ramp * (1 + 0.2 * torch.randn(m, nkv, d, generator=g))).bfloat16().float(),
                       (torch.randn(m, nkv, d, generator=g) * (10.0 ** (torch.arange(m) % 5 - 3))[:, None, None]).bfloat16().float())
        chunk, starts = _chunk(lens, table, loose=loose)
        q = (qs * (0.3 + torch.randn(starts[-1], nkv * G, d, generator=g))).bfloat16()
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        fp.attn_chunk(pool.device(), chunk, q.cuda(), out, scale=scale)
        # int8, more than 64 rows: keys and values in fp16, of which the smallest are off by 2^-25;
        # probabilities below 2^-21 of the largest by 2^-32 of it, times at most all values' magnitudes
        tile = kvq == "int8" and new * G > 64
        floor = 0.0
        if kvq == "int8":
            vmax = max(float(pool.read(table[b], c + n)[1].abs().sum(0).max()) for b, (c, n) in enumerate(lens))
            floor = 2.0 ** -25 + 2.0 ** -32 * vmax
        _check_attention(pool, table, lens, q, out, scale, fp16=tile, floor=floor)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("new,G,d,loose", [(1, 4, 64, 0), (20, 4, 64, 0), (100, 4, 64, 0), (100, 4, 64, 32), (100, 4, 128, 32)])
def test_missing_pages_read_as_zeros_and_take_no_writes(kvq, new, G, d, loose):
    fp = _fp()
    nkv, page, lens = 2, 32, [(200, new), (70, new)]
    g, pool, table = _case(lens, page, nkv, d, kvq, 51)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n)
    for b, i, bad in ((0, 2, -5), (0, 6, 2**31 - 1), (1, 0, pool.n_pages)):
        table[b, i] = bad
    kv = pool.device()
    chunk, starts = _chunk(lens, table, loose=loose)
    N = starts[-1]
    before = [t.clone() for t in ([kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else []))]
    q = torch.randn(N, nkv * G, d, generator=g).bfloat16()
    out = torch.empty(N, nkv * G, d, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(kv, chunk, q.cuda(), out)
    _check_attention(pool, table, lens, q, out)
    # writing over the missing page alone leaves the pool as it was
    gone, s2 = _chunk([(64, 30)], table[:1])
    k = torch.randn(s2[-1], nkv, d, generator=g).bfloat16().cuda()
    fp.kv_append(kv, gone, k, k)
    for a, b in zip(before, [kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else [])):
        assert torch.equal(ref.bits(a), ref.bits(b))
    ko, vo = torch.ones(30, nkv, d, dtype=torch.bfloat16, device="cuda"), torch.ones(30, nkv, d, dtype=torch.bfloat16, device="cuda")
    fp.kv_read(kv, gone, ko, vo)
    assert not ko.any() and not vo.any()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
def test_contents_that_break_the_bounds_stay_inside_the_buffers(kvq):
    """Lengths and rows beyond what the host said: rows past max_new and positions past max_len are
    neither computed nor written; nothing outside the rows and pages changes."""
    fp = _fp()
    nkv, G, d, page = 2, 2, 64, 32
    g, pool, table = _case([(96, 0), (96, 0)], page, nkv, d, kvq, 61, width=3)
    _fill(pool, table, [(96, 0), (96, 0)], g)
    kv = pool.device()
    N = 12
    rs = torch.tensor([2, 9, 400], dtype=torch.int32).cuda()            # 7 rows, then 391 of which 3 exist
    cl = torch.tensor([90, -7], dtype=torch.int32).cuda()
    chunk = fp.Chunk(rs, cl, table.cuda(), max_new=4, max_len=92)       # seq 0: rows 2, 3 at 90, 91; seq 1: 9, 10, 11 at 0, 1, 2
    q = torch.randn(N, nkv * G, d, generator=g).bfloat16()
    out = torch.full((N, nkv * G, d), 7.0, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(kv, chunk, q.cuda(), out)
    seen = [2, 3, 9, 10, 11]
    assert (out[[r for r in range(N) if r not in seen]] == 7.0).all()
    _check_attention(pool, table, [(90, 2), (0, 3)], q[seen], out[seen])
    k, v = (torch.randn(N, nkv, d, generator=g).bfloat16() for _ in range(2))
    fp.kv_append(kv, chunk, k.cuda(), v.cuda())
    pool.write(table[0], torch.tensor([90, 91]), k[2:4].float(), v[2:4].float())
    pool.write(table[1], torch.tensor([0, 1, 2]), k[9:12].float(), v[9:12].float())
    for a, want in zip([kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else []), pool.tensors()):
        assert torch.equal(ref.bits(a.cpu()), ref.bits(want))
    for bad in ([0, 0, 0], [5, 5, 5], [30, 20, 10], [-9, -9, -9]):      # no rows, or rows that run backwards
        rs.copy_(torch.tensor(bad, dtype=torch.int32))
        out.fill_(7.0)
        fp.attn_chunk(kv, chunk, q.cuda(), out)
        fp.kv_append(kv, chunk, k.cuda(), v.cuda())
        assert (out == 7.0).all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
def test_pages_beyond_four_gibytes(kvq):
    fp = _fp()
    nkv, G, d, page = 8, 2, 128, 256
    n_pages = 12000 if kvq == "bf16" else 20000                         # 6.3 and 5.2 GB of keys, as much of values
    kv = fp.PagedKV.empty(n_pages, page, nkv, d, kvq)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2], [7, n_pages - 3, n_pages - 7]], dtype=torch.int32)
    lens = [(600, 70), (500, 1)]
    whole, st = _chunk([(0, c + n) for c, n in lens], table)
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(st[-1], nkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    fp.kv_append(kv, whole, k, v)
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    fp.kv_read(kv, whole, ko, vo)
    if kvq == "bf16":
        assert torch.equal(ko, k) and torch.equal(vo, v)
    for new in ([70, 1], [1, 1]):
        ln = [(c + n - m, m) for (c, n), m in zip(lens, new)]
        chunk, st = _chunk(ln, table)
        q = torch.randn(st[-1], nkv * G, d, generator=g, device="cuda").bfloat16()
        out = torch.empty_like(q)
        fp.attn_chunk(kv, chunk, q, out)
        want, mag = _gpu_attention(kv, table, ln, q)
        assert ((out.double() - want).abs() <= HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * (1 + HALF_BF16)).all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("new", [1, 40])
def test_captured_calls_follow_the_lengths(kvq, new):
    """Append, attention and read back in one graph, replayed with other lengths and rows, eager work of the
    same calls (another workspace) between the replays; two graphs with a workspace each."""
    fp = _fp()
    nkv, G, d, page = 2, 4, 64, 64
    B, width = 3, 40
    g = torch.Generator().manual_seed(71)
    table = ref.tables(g, [width] * B, B * width, width).cuda()
    N = B * new
    qkv = torch.empty(N, (G + 2) * nkv, d, dtype=torch.bfloat16, device="cuda")
    q, k, v = qkv[:, :G * nkv], qkv[:, G * nkv:(G + 1) * nkv], qkv[:, (G + 1) * nkv:]
    cos, sin = (t.cuda() for t in ref.rope_tables(width * page, d))
    rs = torch.arange(0, N + 1, new, dtype=torch.int32).cuda()
    cl = torch.zeros(B, dtype=torch.int32).cuda()
    chunk = fp.Chunk(rs, cl, table, max_new=new)

    def buffers():
        kv = fp.PagedKV.empty(B * width, page, nkv, d, kvq)
        for t in (kv.k, kv.v) + ((kv.k_scales, kv.v_scales) if kvq == "int8" else ()):
            t.zero_()
        return kv, torch.empty(N, G * nkv, d, dtype=torch.bfloat16, device="cuda"), \
            torch.empty(N, G * nkv, d, dtype=torch.bfloat16, device="cuda"), \
            [torch.empty(N, nkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)], fp.attn_chunk_workspace(kv, chunk, N, G * nkv)

    def run(kv, qr, out, kvo, ws):
        fp.kv_append(kv, chunk, k, v, q=q, q_out=qr, cos=cos, sin=sin)
        fp.attn_chunk(kv, chunk, qr, out, workspace=ws)
        fp.kv_read(kv, chunk, *kvo)

    sets = [buffers() for _ in range(3)]
    graphs = []
    for s in sets[:2]:
        run(*s)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            run(*s)
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step, ctx in enumerate([[0, 0, 0], [5, 900, 31], [2000, 17, 64], [63, 2500, 1200], [100, 0, 7]]):
        torch.cuda.synchronize()
        qkv.copy_(torch.randn(qkv.shape, generator=g).bfloat16())
        cl.copy_(torch.tensor(ctx, dtype=torch.int32))
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):            # side by side
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        run(*sets[2])
        torch.cuda.synchronize()
        for s in sets[:2]:
            assert torch.equal(s[2], sets[2][2]) and torch.equal(s[3][0], sets[2][3][0]) and torch.equal(s[3][1], sets[2][3][1]), step
            assert torch.isfinite(s[2].float()).all()


def test_calls_on_other_streams():
    fp = _fp()
    lens = [(700, 3), (40, 60)]
    kv, table, g = _fill_gpu(lens, 64, 2, 64, "int8", 81)
    chunk, st = _chunk(lens, table)
    q = torch.randn(st[-1], 8, 64, generator=g, device="cuda").bfloat16()
    want = torch.empty_like(q)
    fp.attn_chunk(kv, chunk, q, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    a, b = torch.empty_like(q), torch.empty_like(q)
    with pytest.raises(ValueError):
        fp.attn_chunk(kv, chunk, q, a, stream=s)                        # no workspace of its own
    fp.attn_chunk(kv, chunk, q, a, stream=s, workspace=fp.attn_chunk_workspace(kv, chunk, st[-1], 8))
    with torch.cuda.stream(s):
        fp.attn_chunk(kv, chunk, q, b)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want)


def test_strided_rows_and_single_rows():
    """q, k and v as columns of wider rows; one row with an odd stride; unaligned rows are refused."""
    fp = _fp()
    FpError = fp.FpError
    lens = [(50, 1)]
    kv, table, g = _fill_gpu(lens, 32, 2, 64, "bf16", 91)
    chunk, _ = _chunk(lens, table)
    wide = torch.randn(1, 9, 64, generator=g, device="cuda").bfloat16()
    out = torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(kv, chunk, wide[:, 3:7], out)
    want, mag = _gpu_attention(kv, table, lens, wide[:, 3:7])
    assert ((out.double() - want).abs() <= HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * 1.01).all()
    flat = torch.randn(4 * 64 + 1, generator=g, device="cuda").bfloat16()
    with pytest.raises(FpError):
        fp.attn_chunk(kv, chunk, flat[1:].view(1, 4, 64), out)          # 2 bytes off
    with pytest.raises(ValueError):
        fp.attn_chunk(kv, chunk, wide[:, ::2][:, :4], out)              # heads apart
    with pytest.raises(FpError):
        fp.attn_chunk(kv, chunk, out, out)                              # q and out overlap


@pytest.mark.parametrize("loose", [0, 64])
@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,lens", [
    (2, 3, 64, [(40, 5), (200, 1), (31, 2), (0, 4)]),
    (1, 4, 128, [(40, 7), (3000, 8), (95, 1)]),
    (2, 8, 128, [(64, 8), (2000, 5), (25, 7)]),
    (2, 4, 64, [(40, 70), (200, 5), (1500, 130), (90, 1)]),
    (1, 1, 128, [(40, 300), (5, 2), (0, 520)]),
    (1, 16, 128, [(4000, 33)]),
])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(nkv, G, d, lens, kvq, loose):
    fp = _fp()
    page = 64
    g, pool, table = _case(lens, page, nkv, d, kvq, 101)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n)

    def poison(b, pos, dim, x, key=False):
        pg, off = pool._at(table[b], pos)
        h = pos % nkv
        if kvq == "int8":
            (pool.ks if key else pool.vs)[pg, h, off] = x
        elif key:
            pool.k[pg, h, off, dim] = x
        else:
            pool.v[pg, h, off // 32, dim, ref.SLOT[off % 32]] = x

    for b, (c, n) in enumerate(lens):
        if c > 10 and b % 2:
            poison(b, 10, 7, math.inf)                       # in the context: every row sees it
        if n > 1:
            poison(b, c + n // 2, 3, math.nan)
            poison(b, c + n // 2 + (n > 3), d - 1, -math.inf)
            poison(b, c + n - 1, 20, math.inf)
            poison(b, c + n - 1, 5, math.nan, key=True)
    chunk, starts = _chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(pool.device(), chunk, q.cuda(), out)
    want, mag, smag = ref.attention(pool, table, lens, q)
    got = out.cpu().double()
    odd = ~want.isfinite()
    assert odd.any() and not odd.all()
    gn, wn = torch.nan_to_num(got, 1e30, 2e30, 3e30), torch.nan_to_num(want, 1e30, 2e30, 3e30)
    wrong = [(i.tolist(), float(got[tuple(i)]), float(want[tuple(i)])) for i in ((gn != wn) & odd).nonzero()[:8]]
    assert not wrong
    ds = 2 * (d + 4) * EPS32 * smag + (2 * 2.0 ** -11 * smag if kvq == "int8" else 0.0)
    tol = HALF_BF16 * want.abs() + (HALF_BF16 + 2 * ds + 1e-5 + 2.0 ** -11) * mag * (1 + HALF_BF16)
    assert ((got - want).abs() <= tol)[~odd].all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,new,loose", [(2, 2, 64, 1, 0), (1, 8, 128, 4, 0), (2, 8, 64, 6, 0), (2, 4, 128, 50, 64), (2, 4, 64, 50, 64)])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-42, 1e-30])
def test_a_scale_of_nothing_averages(nkv, G, d, new, loose, scale, kvq):
    fp = _fp()
    lens = [(75, new), (0, new), (2100, new)]
    g, pool, table = _case(lens, 64, nkv, d, kvq, 111)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n)
    chunk, starts = _chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(pool.device(), chunk, q.cuda(), out, scale=scale)
    _check_attention(pool, table, lens, q, out, scale, fp16=kvq == "int8")


def _many(B, longest, new, seed, empty=0.1):
    g = torch.Generator().manual_seed(seed)
    ctx = (torch.rand(B, generator=g) ** 3 * longest).int().tolist()
    n = torch.randint(1, new + 1, (B,), generator=g)
    n[torch.rand(B, generator=g) < empty] = 0
    return list(zip(ctx, n.tolist()))


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("B,longest,new,nkv,d", [(64, 300, 1, 2, 64), (65, 300, 90, 1, 128), (200, 100, 3, 2, 64), (1000, 50, 40, 1, 64),
                                                 (4096, 40, 2, 1, 64), (4095, 10, 1, 1, 128)])
def test_many_sequences_append_and_read(B, longest, new, nkv, d, kvq):
    """Rows of every sequence land in its pages and come back; everything else stays as it was."""
    fp = _fp()
    lens = _many(B, longest, new, 121)
    page = 32
    need = [-(-(c + n) // page) for c, n in lens]
    g = torch.Generator(device="cuda").manual_seed(122)
    table = ref.tables(torch.Generator().manual_seed(122), need, sum(need) + 2, max(max(need), 1))
    kv = fp.PagedKV.empty(sum(need) + 2, page, nkv, d, kvq)
    pools = [kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else [])
    for t in pools:
        t.zero_()
    # the whole sequences first, then the new rows over them with other values
    whole, st = _chunk([(0, c + n) for c, n in lens], table)
    k, v = (torch.randn(st[-1], nkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    fp.kv_append(kv, whole, k, v)
    chunk, starts = _chunk(lens, table)
    N = starts[-1]
    k2, v2 = (torch.randn(N + 3, nkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    fp.kv_append(kv, chunk, k2, v2)
    at = torch.cat([torch.arange(st[b] + c, st[b] + c + n) for b, (c, n) in enumerate(lens)]).cuda()
    k[at], v[at] = k2[:N], v2[:N]
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    fp.kv_read(kv, whole, ko, vo)
    k3, v3 = (torch.full_like(t, 7.0) for t in (k2, v2))
    fp.kv_read(kv, chunk, k3, v3)
    assert (k3[N:] == 7.0).all() and (v3[N:] == 7.0).all()
    for got, want in ((ko, k), (vo, v), (k3[:N], k2[:N]), (v3[:N], v2[:N])):
        if kvq == "int8":
            code, scale = ref.quantise(want.float().cpu())
            want = (code.float() * scale.float()[..., None]).bfloat16().cuda()
        assert torch.equal(got, want)


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("B,longest,new,nkv,G,d,kvq", [
    (64, 3000, 1, 2, 4, 64, "bf16"), (65, 9000, 1, 2, 4, 128, "int8"), (200, 2000, 6, 1, 5, 64, "bf16"), (130, 2000, 9, 2, 8, 128, "bf16"),
    (300, 900, 30, 1, 8, 64, "int8"), (100, 4000, 40, 1, 4, 128, "bf16"), (4096, 60, 2, 1, 1, 64, "int8"), (1000, 200, 1, 1, 16, 128, "bf16"),
    (70, 4000, 30, 1, 8, 128, "int8"), (300, 900, 30, 1, 8, 128, "bf16"), (257, 3000, 20, 2, 4, 128, "int8"), (256, 500, 70, 1, 2, 64, "bf16"),
])
def test_many_sequences_attention(B, longest, new, nkv, G, d, kvq, loose):
    fp = _fp()
    if loose and new * G <= 64:
        pytest.skip("the bound changes nothing for so few rows")
    lens = _many(B, longest, new, 131)
    kv, table, g = _fill_gpu(lens, 64, nkv, d, kvq, 131)
    chunk, starts = _chunk(lens, table, loose=64 * loose)
    q = torch.randn(starts[-1] + 1, nkv * G, d, generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    fp.attn_chunk(kv, chunk, q, out)
    assert (out[starts[-1]:] == 7.0).all()
    want, mag = _gpu_attention(kv, table, lens, q[:-1])
    assert ((out[:-1].double() - want).abs() <= HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * (1 + HALF_BF16)).all()


@pytest.mark.parametrize("B", [150, 300])
def test_many_sequences_captured(B):
    """The plan of many sequences is made in the graph, for the lengths at the time of the replay."""
    fp = _fp()
    nkv, G, d, page = 2, 4, 64, 64
    kv, table, g = _fill_gpu([(2500, 0)] * B, page, nkv, d, "int8", 141)
    rs = torch.zeros(B + 1, dtype=torch.int32).cuda()
    cl = torch.zeros(B, dtype=torch.int32).cuda()
    N = 3 * B
    chunk = fp.Chunk(rs, cl, table.cuda(), max_new=3, max_len=2503 // page * page)
    q = torch.randn(N, nkv * G, d, generator=g, device="cuda").bfloat16()
    out, again = torch.zeros_like(q), torch.zeros_like(q)
    ws = fp.attn_chunk_workspace(kv, chunk, N, nkv * G)
    fp.attn_chunk(kv, chunk, q, out, workspace=ws)
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        fp.attn_chunk(kv, chunk, q, out, workspace=ws)
    for seed, longest in ((1, 2400), (2, 30), (3, 700), (4, 2400)):
        lens = _many(B, longest, 3, seed, empty=0.3)
        rs.copy_(torch.tensor([0] + torch.tensor([n for _, n in lens]).cumsum(0).tolist(), dtype=torch.int32))
        cl.copy_(torch.tensor([c for c, _ in lens], dtype=torch.int32))
        q.copy_(torch.randn(N, nkv * G, d, generator=g, device="cuda").bfloat16())
        n = int(rs[-1])
        out.zero_()
        torch.cuda.synchronize()
        gr.replay()
        torch.cuda.synchronize()
        fp.attn_chunk(kv, chunk, q, again)
        assert torch.equal(out[:n], again[:n]) and not out[n:].any()
        want, mag = _gpu_attention(kv, table, lens, q[:n])
        assert ((out[:n].double() - want).abs() <= HALF_BF16 * want.abs() + (HALF_BF16 + 1e-4) * mag * (1 + HALF_BF16)).all()


@pytest.mark.parametrize("nkv,G,d,kvq,lens,bound", [
    (2, 8, 128, "int8", [(1000, 40), (700, 30), (0, 1)], 9600), (2, 8, 128, "int8", [(64, 70)], 9600),
    (2, 8, 128, "bf16", [(1000, 40), (700, 30), (0, 1)], 9600), (1, 16, 128, "bf16", [(2100, 4), (30, 3)], 60000),
    (2, 3, 64, "int8", [(900, 100), (20, 33)], 60000), (2, 3, 64, "bf16", [(900, 100), (20, 33)], 20000),
    (4, 8, 64, "int8", [(900, 6), (1300, 8), (7, 5)], 30000),
])
def test_bounds_of_tiles_of_64_rows(nkv, G, d, kvq, lens, bound):
    """Bounds on the positions for which the call streams in tiles of 64 rows."""
    fp = _fp()
    g, pool, table = _case(lens, 64, nkv, d, kvq, 151)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n)
    table = torch.nn.functional.pad(table, (0, bound // 64 + 1 - table.shape[1]), value=-7)
    chunk, starts = _chunk(lens, table, max_len=bound)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(pool.device(), chunk, q.cuda(), out)
    _check_attention(pool, table, lens, q, out)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("B,max_new,G,d", [(5, 3, 4, 64), (40, 40, 4, 128), (100, 2, 8, 128), (300, 60, 2, 64), (300, 1, 2, 128)])
def test_contents_without_any_order_stay_inside_the_buffers(B, max_new, G, d, kvq):
    """Row starts and contexts of any values at all: rows past the buffers' end and pages of no table keep what
    they hold."""
    fp = _fp()
    nkv, page, width, N, extra = 2, 32, 4, 60, 4
    g = torch.Generator().manual_seed(161)
    big = torch.Generator(device="cuda").manual_seed(161)
    perm = torch.randperm(B * width + 7, generator=g)
    table, spare = perm[:B * width].int().view(B, width), perm[B * width:].cuda()
    kv = fp.PagedKV.empty(B * width + 7, page, nkv, d, kvq)
    pools = [kv.k, kv.v] + ([kv.k_scales, kv.v_scales] if kvq == "int8" else [])
    for t in pools:
        t.fill_(1)
    rs, cl = torch.zeros(B + 1, dtype=torch.int32).cuda(), torch.zeros(B, dtype=torch.int32).cuda()
    around = torch.zeros(B * width + 8192, dtype=torch.int32)          # pages on both sides of the table's
    around[4096:4096 + B * width] = table.flatten()
    held = around.cuda()
    chunk = fp.Chunk(rs, cl, held[4096:4096 + B * width].view(B, width), max_new=max_new, max_len=width * page - 3)
    q, out, k, v, ko, vo = (torch.full((N + extra, h, d), 7.0, dtype=torch.bfloat16, device="cuda") for h in (nkv * G,) * 2 + (nkv,) * 4)
    for t in (q, k, v):
        t[:N] = torch.randn(N, t.shape[1], d, generator=big, device="cuda").bfloat16()
    for lo, hi in ((-20, 100), (0, N + 1), (-2**31, 2**31 - 1), (N - 2, N + 2)):
        rs.copy_(torch.randint(lo, hi, (B + 1,), generator=g).int())
        cl.copy_(torch.randint(max(lo, -2**31), min(4 * hi, 2**31 - 1), (B,), generator=g).int())
        fp.kv_append(kv, chunk, k[:N], v[:N])
        fp.kv_read(kv, chunk, ko[:N], vo[:N])
        fp.attn_chunk(kv, chunk, q[:N], out[:N])
        torch.cuda.synchronize()
        for t in (out, ko, vo):
            assert (t[N:] == 7.0).all()
        for t in pools:
            assert (t[spare] == 1).all()
