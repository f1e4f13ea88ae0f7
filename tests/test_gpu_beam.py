"""Beams on the GPU against the plain 64-bit reference: selection over beams and vocabulary, the caches' change of places, and
a search that uses both."""
import math

import pytest
import torch

import branches_reference as bref
import paged_reference as ref
import test_gpu_paged as paged

pytestmark = pytest.mark.gpu

_fp = paged._fp


def _int(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def _select(logits, scores, done, K, eos=-1, pad=0, stride=None):
    fp = _fp()
    G, W, V = logits.shape
    z = logits.reshape(G * W, V).cuda()
    if stride is not None:                                       # rows of a wider buffer, off 16-byte steps
        w = torch.full((G * W, V + stride), math.nan).cuda()
        w[:, 1:V + 1] = z
        z = w[:, 1:V + 1]
    os, op = torch.full((G, K), 7.0).cuda(), _int([[77] * K] * G)
    oi, od = _int([[77] * K] * G), torch.ones(G, K, dtype=torch.bool).cuda()
    fp.beam_select(z, scores.cuda(), os, op, oi, done=None if done is None else done.cuda(), out_done=od, eos_id=eos, pad_id=pad)
    want = bref.beam_select(logits, scores, done, K, eos, pad)
    assert op.cpu().tolist() == [[c[1] for c in g] for g in want]
    assert oi.cpu().tolist() == [[c[2] for c in g] for g in want]
    assert od.cpu().tolist() == [[c[3] for c in g] for g in want]
    # one rounding to 32 bits of a 64-bit sum
    s = torch.tensor([[c[0] for c in g] for g in want], dtype=torch.float64)
    got, fine = os.cpu().double(), torch.isfinite(s)
    assert torch.equal(got[~fine], s[~fine])
    assert ((got - s).abs()[fine] <= 2.0 ** -24 * s.abs()[fine] * 1.001 + 1e-12).all()
    return want


@pytest.mark.parametrize("G,W,K,V", [(1, 1, 1, 1), (1, 1, 4, 3), (1, 4, 4, 32000), (3, 5, 9, 1000), (2, 1, 16, 4096), (2, 8, 16, 4097),
                                     (70, 2, 3, 50), (1, 64, 64, 300), (1, 33, 64, 9001), (2, 3, 64, 20000), (4, 4, 1, 160001),
                                     (2, 64, 1, 32768), (2, 64, 4, 100000), (2, 16, 32, 70000)])
def test_selection_matches(G, W, K, V):
    g = torch.Generator().manual_seed(G + W + K + V)
    logits = (2.5 * torch.randn(G, 1, V, generator=g) + torch.randn(G, W, V, generator=g))
    scores = -10 - 3 * torch.rand(G, W, generator=g)
    _select(logits, scores, None, K)
    done = torch.rand(G, W, generator=g) < 0.4
    _select(logits, scores, done, K, eos=int(logits[0, 0].argmax()), pad=V + 5, stride=3)
    scores[torch.rand(G, W, generator=g) < 0.3] = -math.inf
    scores[-1, -1] = math.nan
    _select(logits, scores, done, K, eos=2)


def test_equal_scores():
    """Ties go to the lower beam and the lower id: constant logits, beams that are copies, few values."""
    g = torch.Generator().manual_seed(2)
    for W, K, V in ((1, 64, 9000), (4, 64, 9000), (64, 64, 9000), (3, 5, 12), (16, 32, 4096), (64, 64, 70000)):
        same = torch.zeros(2, W, V)
        _select(same, torch.full((2, W), -1.5), None, K)
        row = torch.randn(2, 1, V, generator=g).expand(2, W, V).contiguous()
        _select(row, torch.full((2, W), -1.5), None, K)          # copies
        _select(row.round(), torch.full((2, W), -1.5), None, K)  # few values, many of each
        # (exponentials of one and zero: sums that no order changes)
        few = -800 * torch.randint(0, 3, (2, W, V), generator=g).float()
        _select(few, torch.zeros(2, W), None, K)
        few[:, :, ::2] = -0.0
        _select(few, torch.zeros(2, W), torch.zeros(2, W, dtype=torch.bool), K)


def test_orders_that_fill_few_lanes():
    """Rising and falling logits, all large ones beside each other, or NT ids apart (one thread's): more candidates than are
    ranked at once."""
    V = 3 * 4096 + 77
    i = torch.arange(V).float()
    rows = [i / 100, -i / 100, torch.where((i > 5000) & (i < 6500), i / 50, -i / 1000), torch.where(i % 256 == 3, 50 + i / 500, -i / 1000),
            torch.where(i % 64 == 9, 50 - i / 500, -i / 1000), torch.where(i % 4 == 1, torch.full_like(i, 9.0), i / 5000)]
    logits = torch.stack(rows)[None]
    for K in (1, 7, 64):
        _select(logits, -torch.arange(6.0)[None] / 4, None, K)
        _select(logits.view(6, 1, V), torch.zeros(6, 1), None, K)


def test_masked_and_infinite_logits():
    """Constrained decoding (all but a few ids at -inf or at the type's lowest value), NaN, +inf, rows without any."""
    g = torch.Generator().manual_seed(4)
    G, W, V, K = 3, 6, 10000, 12
    low = torch.finfo(torch.float32).min
    logits = torch.randn(G, W, V, generator=g)
    keep = torch.rand(G, W, V, generator=g) < 0.0003
    for masked in (-math.inf, low, -1e9, math.nan):
        z = torch.where(keep, logits, torch.full_like(logits, masked))
        z[0, 0] = masked
        _select(z, -torch.rand(G, W, generator=g), None, K, eos=5)
    z = logits.clone()
    z[0, 1, [5, 9000]] = math.inf
    z[0, 2] = math.inf
    z[1, :, 17] = math.inf
    z[2, 3] = -math.inf
    z[2, 4, ::2] = math.nan
    z[1, 2] = low
    for K in (3, 12, 64):
        _select(z, -torch.rand(G, W, generator=g), None, K)
        _select(z, torch.full((G, W), -1.0), torch.tensor([[True, False, True, False, False, False]] * G), K)
    _select(torch.full((2, 3, 20), -math.inf), torch.zeros(2, 3), None, 4)
    _select(z, torch.full((G, W), -math.inf), None, 4)


def test_the_largest_vocabulary():
    g = torch.Generator().manual_seed(6)
    V = 1 << 20
    z = torch.randn(1, 2, V, generator=g)
    _select(z, torch.tensor([[-1.0, -1.1]]), None, 20)
    _select(torch.zeros(1, 2, V), torch.tensor([[-1.0, -1.0]]), None, 20)
    z[0, 1] = z[0, 1, 0]
    z[0, 1, V - 1] += 1
    _select(z, torch.tensor([[-1.0, -1.1]]), None, 64)


def test_selection_refuses_other_shapes():
    fp = _fp()
    z, s = torch.zeros(6, 9).cuda(), torch.zeros(2, 3).cuda()
    os, oi = torch.zeros(2, 4).cuda(), _int([[0] * 4] * 2)
    op, od = oi.clone(), torch.zeros(2, 4, dtype=torch.bool).cuda()
    fp.beam_select(z, s, os, op, oi, out_done=od)
    for bad in (dict(logits=z[:5]), dict(scores=s.double()), dict(out_scores=os[:, :3]), dict(out_parent=op.long()), dict(done=s),
                dict(out_done=od.int()), dict(logits=z.t()), dict(done=od), dict(stream=torch.cuda.Stream())):
        a = dict(logits=z, scores=s, out_scores=os, out_parent=op, out_ids=oi)
        a.update(bad)
        with pytest.raises(ValueError):
            fp.beam_select(**a)
    with pytest.raises(fp.FpError):
        fp.beam_select(z, s, os, op, oi, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


# ------------------------------------------------------------------ caches
def _pool(n_pages, page, nkv, d, kvq, g):
    """A pool with random bits on every position."""
    p = ref.Pool(n_pages, page, nkv, d, kvq)
    for t in p.tensors():
        t.copy_(torch.randint(-100, 100, t.shape, generator=g).to(t.dtype))
    return p


def _reordered(pools, table, lens, parent, page, W):
    """Tables and pools after the call; pools' positions behind a sequence's last are not looked at."""
    tab, copies = [], []
    for i, n in enumerate(lens):
        new, c = bref.reorder(table[i * W:(i + 1) * W].tolist(), n, parent[i], page, W)
        tab += new
        copies += [(a, b, n % page) for a, b in c]
    return torch.tensor(tab, dtype=torch.int32), copies


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("nkv,d,page,W,lens", [
    (2, 64, 32, 4, [5, 32, 0, 70, 95]), (3, 128, 96, 1, [40, 96]), (1, 64, 64, 64, [200, 33]), (4, 128, 256, 7, [300, 255, 257]),
    (8, 64, 32, 5, [31] * 40), (1, 128, 160, 33, [801, 160]),
])
def test_reordering_matches(nkv, d, page, W, lens, in_place):
    fp = _fp()
    g = torch.Generator().manual_seed(W + page)
    G = len(lens)
    need = [n + 2 * page for n in lens for _ in range(W)]
    per = [-(-n // page) for n in need]
    table = ref.tables(g, per, sum(per) + 2, max(per) + 1)
    pools = [_pool(sum(per) + 2, page, nkv, d, q, g) for q in ("bf16", "int8", "int8")]
    parent = torch.randint(0, W, (G, W), generator=g)
    parent[0] = W - 1                                            # all from one
    if G > 1:
        parent[1] = torch.arange(W).flip(0)                      # everyone from another
    if G > 2:
        parent[2, 0], parent[2, -1] = -1, 2**31 - 1              # out of range: itself
    kvs = [p.device() for p in pools]
    tab = table.cuda()
    out = tab if in_place else torch.full_like(tab, 77)
    ctx = _int([n for n in lens for _ in range(W)])
    fp.beam_reorder(kvs, tab, ctx, parent.int().cuda(), table_out=None if in_place else out)
    want, copies = _reordered(pools, table, lens, parent.tolist(), page, W)
    assert torch.equal(out.cpu(), want)
    if not in_place:
        assert torch.equal(tab.cpu(), table)
    for kv, pool in zip(kvs, pools):
        k, v = pool.k.clone(), pool.v.clone()
        sc = [t.clone() for t in (pool.ks, pool.vs)] if pool.kvq == "int8" else []
        hidden = torch.zeros(pool.n_pages, page, dtype=torch.bool)       # positions behind the last of a copied page's
        for a, b, n in copies:
            hidden[b, n:] = True
            k[b, :, :n] = pool.k[a, :, :n]
            pos = torch.arange(n)
            v[b, :, pos // 32, :, ref.SLOT[pos % 32]] = pool.v[a, :, pos // 32, :, ref.SLOT[pos % 32]]
            for t, o in zip(sc, (pool.ks, pool.vs)):
                t[b, :, :n] = o[a, :, :n]
        see = ~hidden
        pg, off = see.nonzero(as_tuple=True)
        for a, w in ((kv.k, k), (kv.k_scales, sc[0] if sc else None), (kv.v_scales, sc[1] if sc else None)):
            if w is not None:
                assert torch.equal(ref.bits(a.cpu()[pg, :, off].contiguous()), ref.bits(w[pg, :, off].contiguous()))
        sl = ref.SLOT[off % 32]
        assert torch.equal(ref.bits(kv.v.cpu()[pg, :, off // 32, :, sl].contiguous()), ref.bits(v[pg, :, off // 32, :, sl].contiguous()))


def test_reordering_with_missing_pages_and_odd_lengths():
    """A missing last page reads as zeros and takes no copy; lengths past the table, or below zero, copy nothing."""
    fp = _fp()
    g = torch.Generator().manual_seed(3)
    page, W, nkv, d = 32, 3, 2, 64
    pool = _pool(20, page, nkv, d, "bf16", g)
    table = torch.arange(18, dtype=torch.int32).view(6, 3)
    table[1, 1], table[4, 1] = -3, 99                            # group 0: beam 1's; group 1: beam 1's
    kv, tab = pool.device(), table.cuda()
    # group 0: beam 2 goes on from beam 1, whose page is missing: zeros into free beam 0's; group 1: beam 1's is the free one
    fp.beam_reorder(kv, tab, _int([40] * 6), _int([[1, 2, 1], [0, 0, 2]]))
    want, _ = _reordered([pool], table, [40, 40], [[1, 2, 1], [0, 0, 2]], page, W)
    assert torch.equal(tab.cpu(), want)
    k = pool.k.clone()
    k[1] = 0                                                     # page table[0][1]
    got = kv.k.cpu()
    assert torch.equal(got[1, :, :8], k[1, :, :8])
    rest = [i for i in range(20) if i != 1]
    assert torch.equal(got[rest], k[rest])
    for n in (96, 200, 2**31 - 1, -5, 0):
        kv, tab = pool.device(), table.cuda()
        fp.beam_reorder(kv, tab, _int([n] * 6), _int([[1, 1, 1], [2, 2, 2]]))
        full = max(0, min(3, n // page))
        exp = table.clone()
        exp[:3, :full], exp[3:, :full] = table[1, :full], table[5, :full]
        assert torch.equal(tab.cpu(), exp) and torch.equal(kv.k.cpu(), pool.k)


def test_a_search_keeps_every_beam_its_history():
    """Selection, reordering and appends over many steps and pages: what each beam's cache holds is what its tokens
    wrote.  Pages that no row names any more are handed out again."""
    fp = _fp()
    g = torch.Generator().manual_seed(8)
    G, W, V, page, nkv, d, steps, P = 3, 5, 200, 32, 2, 64, 80, 20
    width = -(-(P + steps) // page)
    n_pages = G * W * (width + 1)
    kvs = [fp.PagedKV.empty(n_pages, page, nkv, d, "bf16") for _ in range(2)]
    words = torch.randn(2, V, 2, nkv, d, generator=g).bfloat16().cuda()     # a token's key and value in each layer
    prompt = torch.randint(V, (G, P), generator=g).cuda()
    B = G * W
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[:, 0] = torch.arange(B)
    table, ctx = table.cuda(), _int([0] * B)
    one = torch.arange(B + 1, dtype=torch.int32).cuda()
    chunk = fp.Chunk(one, ctx, table, max_new=1, max_len=P + steps)
    # the prompt goes to every group's first beam
    first = fp.Chunk(_int([0, P, P, P, P, P, 2 * P, 2 * P, 2 * P, 2 * P, 2 * P, 3 * P, 3 * P, 3 * P, 3 * P, 3 * P]), ctx, table, max_new=P, max_len=P + steps)
    for kv, w in zip(kvs, words):
        fp.kv_append(kv, first, w[prompt.view(-1), 0].contiguous(), w[prompt.view(-1), 1].contiguous())
    hist = prompt[:, None].expand(G, W, P).clone()
    scores, done = torch.zeros(G, W, device="cuda"), torch.zeros(G, W, dtype=torch.bool, device="cuda")
    os, od = torch.empty_like(scores), torch.empty_like(done)
    op, oi = torch.empty(G, W, dtype=torch.int32, device="cuda"), torch.empty(G, W, dtype=torch.int32, device="cuda")
    z1 = torch.randn(G, V, generator=g).cuda()
    fp.beam_select(z1, scores[:, :1].contiguous(), os, op, oi)             # a request's first step
    assert (op == 0).all()
    ctx.fill_(P)
    for step in range(steps):
        fp.beam_reorder(kvs, table, ctx, op)
        hist = torch.cat([hist.gather(1, op.long()[..., None].expand(G, W, hist.shape[-1])), oi.long()[..., None]], -1)
        scores.copy_(os)
        n = int(ctx[0])
        if n % page == 0:                                                  # the host hands out pages nobody has
            used = set(table[:, :n // page].flatten().tolist())
            fresh = [p for p in range(n_pages) if p not in used][:B]
            table[:, n // page] = _int(fresh)
        for kv, w in zip(kvs, words):
            fp.kv_append(kv, chunk, w[oi.view(-1).long(), 0].contiguous(), w[oi.view(-1).long(), 1].contiguous())
        ctx += 1
        z = (2 * torch.randn(G * W, V, generator=g)).cuda()
        fp.beam_select(z, scores, os, op, oi)
        if step % 7 == 6 or step == steps - 1:
            n = int(ctx[0])
            whole = fp.Chunk(torch.arange(0, (B + 1) * n, n, dtype=torch.int32).cuda(), _int([0] * B), table, max_new=n, max_len=P + steps)
            for kv, w in zip(kvs, words):
                k, v = (torch.empty(B * n, nkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
                fp.kv_read(kv, whole, k, v)
                t = hist.reshape(-1)
                assert torch.equal(k, w[t, 0]) and torch.equal(v, w[t, 1]), step
    assert len({tuple(h) for h in hist.view(B, -1).tolist()}) == B


def test_captured_beams_follow_their_contents():
    """Selection and reordering in one graph, replayed with other logits, lengths and finished beams, eager work of the same calls
    between the replays; two graphs with a workspace each."""
    fp = _fp()
    g = torch.Generator().manual_seed(17)
    G, W, V, page, nkv, d = 2, 4, 5000, 32, 2, 64
    table = torch.arange(G * W * 4, dtype=torch.int32).view(G * W, 4)
    pool = _pool(G * W * 4, page, nkv, d, "int8", g)

    class Side:
        def __init__(self):
            self.kv, self.table, self.out = pool.device(), table.cuda(), torch.empty_like(table).cuda()
            self.ctx = _int([0] * (G * W))
            self.lg, self.scores = torch.zeros(G * W, V).cuda(), torch.zeros(G, W).cuda()
            self.done, self.od = (torch.zeros(G, W, dtype=torch.bool).cuda() for _ in range(2))
            self.os, self.op, self.oi = torch.zeros(G, W).cuda(), _int([[0] * W] * G), _int([[0] * W] * G)
            self.ws = fp.beam_select_workspace(G, W, W, V)

        def run(self):
            fp.beam_select(self.lg, self.scores, self.os, self.op, self.oi, done=self.done, out_done=self.od, eos_id=3, workspace=self.ws)
            fp.beam_reorder([self.kv], self.table, self.ctx, self.op, table_out=self.out)
            self.table.copy_(self.out)

        def state(self):
            return [self.os, self.op, self.oi, self.od, self.table, self.kv.k, self.kv.v, self.kv.k_scales]

    sides = [Side() for _ in range(3)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for s in sides[:2]:
        s.run()
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            s.run()
        graphs.append(gr)
    sides[2].run()
    for it, n in enumerate([5, 40, 64, 97, 31, 100]):
        data = {"lg": 3 * torch.randn(G * W, V, generator=g), "scores": -torch.rand(G, W, generator=g), "ctx": torch.full((G * W,), n, dtype=torch.int32),
                "done": torch.rand(G, W, generator=g) < 0.3}
        if it == 3:
            data["lg"].zero_()
        for s in sides:
            for name, t in data.items():
                getattr(s, name).copy_(t.cuda())
        torch.cuda.synchronize()
        sides[2].run()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for s in sides[:2]:
            for a, b in zip(s.state(), sides[2].state()):
                assert torch.equal(ref.bits(a), ref.bits(b)), it


def test_beams_on_another_stream():
    """On a stream of the caller's, with a workspace of its own; without one another stream is refused."""
    fp = _fp()
    G, W, V, page = 2, 4, 5000, 32
    g = torch.Generator().manual_seed(8)
    z, s = torch.randn(G * W, V, generator=g).cuda(), torch.randn(G, W, generator=g).cuda()
    kv = fp.PagedKV.empty(20, page, 2, 64, "int8")
    for t in (kv.k, kv.v):
        t.random_(-127, 127)
    for t in (kv.k_scales, kv.v_scales):
        t.uniform_(0.1, 1)
    start = [t.clone() for t in (kv.k, kv.v, kv.k_scales, kv.v_scales)]
    ctx, st = _int([40] * G * W), torch.cuda.Stream()
    ws = fp.beam_select_workspace(G, W, W, V)
    got = []
    for stream in (None, st):
        for t, x in zip((kv.k, kv.v, kv.k_scales, kv.v_scales), start):
            t.copy_(x)
        os, op, oi, table = torch.zeros(G, W).cuda(), _int([[7] * W] * G), _int([[7] * W] * G), _int([[2 * i, 2 * i + 1] for i in range(G * W)])
        torch.cuda.synchronize()
        fp.beam_select(z, s, os, op, oi, workspace=ws, stream=stream)
        fp.beam_reorder(kv, table, ctx, op, stream=stream)
        torch.cuda.synchronize()
        got.append([os, op, oi, table] + [t.clone() for t in (kv.k, kv.v, kv.k_scales, kv.v_scales)])
    for a, b in zip(*got):
        assert torch.equal(ref.bits(a.cpu()), ref.bits(b.cpu()))
    with pytest.raises(ValueError, match="workspace"):
        fp.beam_select(z, s, os, op, oi, stream=st)


def test_scores_that_differ_beyond_12_digits():
    """Beams whose sums of exponentials differ by some 5e-13 of themselves are told apart, whichever comes first: a row of n logits
    a below one of zero has log(1 + n e^a).  The roundings of such a sum of some thousand 64-bit numbers, of its 64-bit
    exponentials and of its logarithm stay below 1e-14."""
    from decimal import Decimal, localcontext
    rows = [(1081, -2.3070878982543945, 1342, -2.523362398147583), (2162, -2.3503623008728027, 2684, -2.566636800765991),
            (2829, -2.328671455383301, 1957, -1.9601608514785767), (3929, -2.3936831951141357, 1922, -1.6786645650863647),
            (3929, -1.9387843608856201, 1922, -1.2237657308578491), (1081, -1.202321171760559, 1342, -1.4185956716537476)]
    fp = _fp()
    for V in (4096, 9001):
        for n0, a0, n1, a1 in rows:
            z = torch.full((1, 2, V), -math.inf)
            for w, (n, a) in enumerate(((n0, a0), (n1, a1))):
                z[0, w, :1] = 0.0
                z[0, w, V - n:] = a
            with localcontext() as c:
                c.prec = 40
                lse = [(1 + n * Decimal(float(z[0, w, -1])).exp()).ln() for w, n in enumerate((n0, n1))]
            assert 4e-13 < lse[0] - lse[1] < 1e-12
            for turn in (0, 1):
                o, p, i = torch.empty(1, 2).cuda(), _int([[7, 7]]), _int([[7, 7]])
                fp.beam_select((z.flip(1) if turn else z)[0].contiguous().cuda(), torch.zeros(1, 2).cuda(), o, p, i)
                assert i.tolist() == [[0, 0]]
                assert p.tolist() == ([[0, 1]] if turn else [[1, 0]]), (V, n0, a0, turn)
