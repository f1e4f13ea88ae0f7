"""Chunk attention at the ends of the number ranges that its entry accepts."""
import math

import pytest
import torch

import paged_reference as ref
import test_gpu_paged as paged

pytestmark = pytest.mark.gpu

# (rows of every tile size; with a loose bound more than 64 rows take the tiles of 256)
CALLS = [(1, 8, 1, 0), (2, 8, 5, 0), (2, 4, 60, 0), (2, 4, 60, 64), (1, 1, 300, 64)]


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,new,loose", CALLS)
@pytest.mark.parametrize("size", [1e-30, 1e-10, 1e-8, 1e-6, 1e-3, 1e6, 1e30])
def test_queries_of_any_size(size, nkv, G, new, loose, kvq):
    """Queries of one size and a scale that makes ordinary scores of them; rows of zeros and rows 2^20 smaller
    beside them."""
    fp = paged._fp()
    d, page, lens = 128, 64, [(900, new), (70, new)]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 171)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = size * torch.randn(starts[-1], nkv * G, d, generator=g)
    q[1::5] = 0
    q[3::5] *= 2.0 ** -20
    q = q.bfloat16()
    scale = 2.0 / math.sqrt(d) / size
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(pool.device(), chunk, q.cuda(), out, scale=scale)
    # int8 in tiles of 256 rows: keys, values and queries meet the matrix cores as fp16
    paged._check_attention(pool, table, lens, q, out, scale, fp16=kvq == "int8" and bool(loose))


@pytest.mark.parametrize("nkv,G,d,lens,loose", [
    (1, 8, 128, [(900, 1), (5000, 1)], 0), (2, 8, 64, [(3000, 3), (31, 4)], 0), (2, 4, 128, [(300, 20), (0, 64)], 0),
    (2, 4, 128, [(2000, 64), (0, 300)], 64), (1, 2, 64, [(700, 200), (5, 1)], 64), (1, 1, 128, [(0, 1000)], 64),
])
@pytest.mark.parametrize("top", [2.0 ** 126, 2.0 ** 112, 2.0 ** -60])
def test_values_of_any_size(top, nkv, G, d, lens, loose):
    """bf16 values of one sign, so that nothing cancels in the sums: finite outputs for all that are below 2^127."""
    fp = paged._fp()
    page = 64
    g, pool, table = paged._case(lens, page, nkv, d, "bf16", 181)
    for b, (c, n) in enumerate(lens):
        m = c + n
        pool.write(table[b], torch.arange(m), torch.randn(m, nkv, d, generator=g).bfloat16().float(),
                   (top * (0.5 + 0.5 * torch.rand(m, nkv, d, generator=g))).bfloat16().float())
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(pool.device(), chunk, q.cuda(), out)
    assert torch.isfinite(out.float()).all()
    paged._check_attention(pool, table, lens, q, out)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,new,loose", CALLS)
def test_scales_of_any_size(nkv, G, new, loose, kvq):
    """The largest scales, with queries of zeros (whose scores are zero) and queries whose scores lie some hundred
    apart; beyond 2^127 the scale to base 2 would pass fp32's largest number, and is refused."""
    fp = paged._fp()
    d, page, lens = 128, 64, [(900, new), (70, new)]
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 175)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = 2.0 ** -123 * torch.randn(starts[-1], nkv * G, d, generator=g)
    q[::3] = 0
    q = q.bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    # int8: a probability (streamed: times its value's scale) enters the product as fp16, where it is off by up to 2^-25
    # however small it is.  The row's largest is held at 2^7 or more (streamed: 2^7 over the largest scale) and the quotient's
    # lower side is at least that: 2^-32 of the largest value for each key
    n = max(c + m for c, m in lens)
    floor = 2.0 ** -32 * n * max(float(pool.read(table[b], c + m)[1].abs().max()) for b, (c, m) in enumerate(lens)) * 1.01
    floor = floor if kvq == "int8" else 0.0
    for scale in (2.0 ** 127 * (1 - 2.0 ** -24), -2.0 ** 126):
        fp.attn_chunk(pool.device(), chunk, q.cuda(), out, scale=scale)
        paged._check_attention(pool, table, lens, q, out, scale, fp16=kvq == "int8" and bool(loose), floor=floor)
    for scale in (2.0 ** 127, -3.3e38):
        with pytest.raises(fp.FpError):
            fp.attn_chunk(pool.device(), chunk, q.cuda(), out, scale=scale)


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("d,new", [(64, 1), (64, 70), (128, 300)])
def test_the_longest_sequence(d, new, kvq):
    """A sequence of the most positions that a call takes, nearly all of them in one shared page whose scores are far
    below those of the last page; what lies behind its end is NaN."""
    fp = paged._fp()
    page, length = 65536, 2 ** 31 - 1024
    last = length - 32767 * page                       # positions in the last page
    pool = ref.Pool(2, page, 1, d, kvq)
    g = torch.Generator().manual_seed(177)
    two = torch.tensor([0, 1], dtype=torch.int32)
    pool.write(two, torch.arange(page), torch.full((page, 1, d), -8.0), torch.full((page, 1, d), 5.0))
    k, v = (torch.randn(last, 1, d, generator=g).bfloat16().float() for _ in range(2))
    pool.write(two, page + torch.arange(last), k, v)
    table = torch.zeros(1, 32768, dtype=torch.int32)
    table[0, -1] = 1
    kv = pool.device()
    chunk = fp.Chunk(torch.tensor([0, new], dtype=torch.int32).cuda(), torch.tensor([length - new], dtype=torch.int32).cuda(),
                     table.cuda(), max_new=new)
    q = (1 + 0.25 * torch.rand(new, 2, d, generator=g)).bfloat16()
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    fp.attn_chunk(kv, chunk, q.cuda(), out)
    # the shared page's scores are below -8 sqrt(d), the last page's largest above 0: 2^31 times e^-64 is nothing
    kd, vd = (t[page:, 0].cuda() for t in pool.read(two, page + last))
    seen = last - new + 1 + torch.arange(new, device="cuda")
    for h in range(2):
        s = q[:, h].cuda().double() @ kd.t().contiguous() / math.sqrt(d)
        s.masked_fill_(torch.arange(last, device="cuda")[None, :] >= seen[:, None], -math.inf)
        p = torch.softmax(s, -1)
        want, mag = p @ vd, p @ vd.abs()
        err = (out[:, h].double() - want).abs()
        # roundings of the output and the probabilities; int8 in tiles of 256 rows: keys and values in fp16, a key's share of
        # the score on both sides of the quotient; fp32 scores and sums below 1e-3
        smag = float((q[:, h].cuda().double().abs() @ kd.abs().t().contiguous()).max()) / math.sqrt(d)
        f16 = 2.0 ** -11 * (1 + 2 * smag) if kvq == "int8" else 0.0
        assert (err <= paged.HALF_BF16 * want.abs() + (paged.HALF_BF16 + f16 + 1e-3) * mag * 1.01).all()
    # the rows' own positions, written and read back across the last blocks
    rows = torch.randn(new, 1, d, generator=g).bfloat16().cuda()
    fp.kv_append(kv, chunk, rows, rows)
    ko, vo = torch.empty_like(rows), torch.empty_like(rows)
    fp.kv_read(kv, chunk, ko, vo)
    want = rows
    if kvq == "int8":
        code, scale = ref.quantise(rows.float().cpu())
        want = (code.float() * scale.float()[..., None]).bfloat16().cuda()
    assert torch.equal(ko, want) and torch.equal(vo, want)


def test_rows_of_the_widest_buffer():
    """Two sequences' next tokens in row buffers of 2^24 rows: the launch goes by the rows that they can own."""
    fp = paged._fp()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 70 GB")
    nkv, G, d, lens = 8, 2, 64, [(200, 1), (31, 1)]
    kv, table, g = paged._fill_gpu(lens, 64, nkv, d, "bf16", 179)
    chunk, starts = paged._chunk(lens, table)
    q = torch.empty(1 << 24, nkv * G, d, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    q[:2] = torch.randn(2, nkv * G, d, generator=g, device="cuda").bfloat16()
    out[:4] = 7.0
    out[-1] = 7.0
    fp.attn_chunk(kv, chunk, q, out)
    want, mag = paged._gpu_attention(kv, table, lens, q[:2])
    got, untouched = out[:2].double(), (out[2:4] == 7.0).all() and (out[-1] == 7.0).all()
    del q, out
    torch.cuda.empty_cache()
    assert ((got - want).abs() <= paged.HALF_BF16 * want.abs() + (paged.HALF_BF16 + 1e-4) * mag * 1.01).all()
    assert untouched
