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


def _chunk(lens, table, extra_rows=0, max_len=None, max_new=None):
    fp = _fp()
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
def _check_attention(pool, table, lens, q, out, scale=None):
    want, mag, smag = ref.attention(pool, table, lens, q, scale)
    N = want.shape[0]
    d = q.shape[2]
    # output rounding; probabilities rounded to bf16 before they meet v (their sum is not); fp32
    # scores of d products, each side of the quotient off by the largest score error
    ds = 2 * (d + 4) * EPS32 * smag
    tol = HALF_BF16 * want.abs() + (HALF_BF16 + 2 * ds + 1e-5) * mag * (1 + HALF_BF16)
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


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,page", SHAPES)
@pytest.mark.parametrize("seqs", sorted(ATTN_SEQS))
def test_attention_matches_the_reference(seqs, nkv, G, d, page, kvq):
    fp = _fp()
    lens = ATTN_SEQS[seqs]
    g, pool, table = _case(lens, page, nkv, d, kvq, 21)
    _fill(pool, table, lens, g, upto=lambda c, n: c + n, scale=1.5)
    kv = pool.device()
    chunk, starts = _chunk(lens, table)
    N = starts[-1]
    q = torch.randn(N + 2, nkv * G, d, generator=g).bfloat16()
    out = torch.full((N + 2, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda()
    fp.attn_chunk(kv, chunk, q.cuda(), out)
    assert (out[N:] == 7.0).all()
    _check_attention(pool, table, lens, q[:N], out)
    again = torch.empty_like(out)
    fp.attn_chunk(kv, chunk, q.cuda(), again)
    assert torch.equal(ref.bits(again[:N]), ref.bits(out[:N]))
