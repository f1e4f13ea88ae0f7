"""Keys and values that are not finite on their way into an int8 cache and out of it, and the time that
unwritten positions may take."""
import math

import pytest
import torch

import paged_reference as ref
import test_gpu_paged as paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("nkv,G,d,lens,loose", [
    (2, 4, 64, [(40, 3), (31, 5)], 0), (3, 2, 128, [(100, 40), (0, 33)], 0), (1, 4, 128, [(300, 70), (5, 64)], 64),
])
def test_int8_appends_of_values_that_are_not_finite(nkv, G, d, lens, loose, rotated):
    """A position and kv head with a NaN, an infinity or a magnitude that the scale cannot hold reads back as NaN
    throughout, as fp16(absmax / 127) and rint(x / s) have it, and the rows that see it are NaN; all others are
    what they are without it."""
    fp = paged._fp()
    page = 64
    g, pool, table = paged._case(lens, page, nkv, d, "int8", 191)
    paged._fill(pool, table, lens, g)
    chunk, starts = paged._chunk(lens, table)
    seen, _ = paged._chunk(lens, table, loose=loose)
    N = starts[-1]
    k, v, q = (torch.randn(N, h, d, generator=g).bfloat16() for h in (nkv, nkv, nkv * G))
    sick = {"k": torch.zeros(N, nkv, dtype=torch.bool), "v": torch.zeros(N, nkv, dtype=torch.bool)}
    kinds = [math.nan, math.inf, -math.inf, 1e9, -1e30]
    for b, (c, n) in enumerate(lens):
        for i, x in enumerate(kinds):
            r, t, name = starts[b] + n - 1 - i % max(1, n // 2), (k, v)[(b + i) % 2], "kv"[(b + i) % 2]
            t[r, (b + i) % nkv, (7 * i + (d // 2 if i % 2 else 3)) % d] = x
            sick[name][r, (b + i) % nkv] = True
    v[starts[1] - 1, 0] = math.nan                      # all of it
    sick["v"][starts[1] - 1, 0] = True
    cos, sin = ref.rope_tables(max(c + n for c, n in lens), d)
    args = dict(q=q.cuda(), q_out=torch.empty_like(q, device="cuda"), cos=cos.cuda(), sin=sin.cuda()) if rotated else {}

    def run(k, v):
        kv = pool.device()
        fp.kv_append(kv, chunk, k.cuda(), v.cuda(), **args)
        ko, vo = (torch.empty(N, nkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        fp.kv_read(kv, chunk, ko, vo)
        out = torch.empty(N, nkv * G, d, dtype=torch.bfloat16, device="cuda")
        fp.attn_chunk(kv, seen, q.cuda(), out)
        return ko.cpu(), vo.cpu(), out.cpu(), kv

    clean = run(*[torch.where(sick[n][..., None], torch.ones_like(t), t) for t, n in ((k, "k"), (v, "v"))])
    ko, vo, out, kv = run(k, v)
    for got, want, bad in ((ko, clean[0], sick["k"]), (vo, clean[1], sick["v"])):
        assert torch.isnan(got[bad]).all()
        assert torch.equal(got[~bad], want[~bad])
    for s, bad in ((kv.k_scales, sick["k"]), (kv.v_scales, sick["v"])):
        for b, (c, n) in enumerate(lens):
            pos = torch.arange(c, c + n)
            pg, off = pool._at(table[b], pos)
            assert torch.equal(s.cpu()[pg, :, off].isfinite(), ~bad[starts[b]:starts[b + 1]])
    # rows up to the first such position of their kv head are as without it, the later ones NaN
    for b, (c, n) in enumerate(lens):
        rows = slice(starts[b], starts[b + 1])
        reach = (sick["k"] | sick["v"])[rows].cumsum(0) > 0
        reach = reach.repeat_interleave(G, 1)
        assert torch.isnan(out[rows][reach]).all()
        # (probabilities meet the values as fp16 relative to the block's largest scale, which the two runs differ
        # in: 2^-11 of the values' sum either way, fp32 sums, and both outputs' rounding)
        a, w = out[rows][~reach].double(), clean[2][rows][~reach].double()
        assert ((a - w).abs() <= 2 * (paged.HALF_BF16 * w.abs() * 1.01 + (2.0 ** -11 + 1e-5) * 1.01 * clean[1].abs().amax())).all()


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("nkv,G,d,lens,loose", [
    (2, 4, 128, [(1500, 301), (0, 333)], 64),           # tiles of 256 rows
    (2, 4, 64, [(1500, 301), (0, 333)], 64),
    (2, 4, 64, [(0, 75)] * 4, 0),                       # streamed
    (4, 8, 128, [(2000, 17)] * 8, 0),
])
def test_what_unwritten_positions_hold_takes_no_time(nkv, G, d, lens, loose, kvq):
    """Sequences that end inside a block: NaN behind their ends costs nothing against zeros there.  (Looking
    at each position again for each row costs tens of times the whole call.)"""
    fp = paged._fp()
    page = 64
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 201)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16().cuda()
    odd = pool.device()
    plain = [t.clone() for t in pool.tensors()]
    if kvq == "bf16":
        plain = [torch.nan_to_num(t, 0.0) for t in plain]
    else:
        plain[2:] = [torch.nan_to_num(t, 0.0) for t in plain[2:]]
    even = fp.PagedKV(*[t.cuda() for t in plain])
    out = {}
    ws = fp.attn_chunk_workspace(odd, chunk, starts[-1], nkv * G)

    def us(kv, name):
        out[name] = torch.empty_like(q)
        best = math.inf
        for _ in range(12):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            fp.attn_chunk(kv, chunk, q, out[name], workspace=ws)
            b.record()
            b.synchronize()
            best = min(best, 1e3 * a.elapsed_time(b))
        return best

    te, to = us(even, "even"), us(odd, "odd")
    assert torch.equal(out["even"], out["odd"])
    assert to < 2 * te, f"{to:.0f} us with NaN, {te:.0f} us with zeros"
