"""Verification of drafted tokens on the GPU against the row-by-row 64-bit reference: the same tokens,
exactly."""
import math

import pytest
import torch

import paged_reference as ref

pytestmark = pytest.mark.gpu


def _run(logits, starts, ids, probs, u, ul, T, max_rows, stride=None):
    import paper_2501_13111_amd as fp
    B, (N, V) = len(starts) - 1, logits.shape

    def wide(t):                                     # rows of a wider buffer, off 16-byte steps
        if stride is None:
            return t.cuda()
        w = torch.full((N, V + stride), math.nan)
        w[:, 1:V + 1] = t
        return w.cuda()[:, 1:V + 1]

    out = torch.full((B, max_rows), 77, dtype=torch.int32).cuda()
    n = torch.full((B,), 77, dtype=torch.int32).cuda()
    fp.verify_draft(wide(logits), torch.tensor(starts, dtype=torch.int32).cuda(), ids.cuda(), u.cuda(), ul.cuda(), out, n,
                    draft_probs=None if probs is None else wide(probs), temperature=T)
    want = ref.verify(logits, starts, ids, probs, u, ul, T, max_rows)
    exp = torch.full((B, max_rows), -1, dtype=torch.int32)
    for b, t in enumerate(want):
        exp[b, :len(t)] = torch.tensor(t, dtype=torch.int32)
    assert n.cpu().tolist() == [len(t) for t in want]
    assert torch.equal(out.cpu(), exp)
    return want


def _inputs(g, rows, V, T, with_probs, noise=0.4):
    N = sum(rows)
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    logits = 2 * torch.randn(N, V, generator=g)
    near = logits + noise * torch.randn(N, V, generator=g)
    if with_probs and T > 0:
        probs = torch.softmax(near.double() / T, -1).float()
        ids = torch.multinomial(probs, 1, generator=g)[:, 0].int()
    else:
        probs, ids = None, near.argmax(-1).int()
    return starts, logits, probs, ids, torch.rand(N, generator=g), torch.rand(len(rows), generator=g)


@pytest.mark.parametrize("T", [0.0, 0.3, 1.0, 2.5])
@pytest.mark.parametrize("with_probs", [False, True])
@pytest.mark.parametrize("rows,V", [([1], 1), ([4], 17), ([2, 1, 5, 3], 1000), ([6] * 9, 4096), ([3, 0, 2], 4097),
                                    ([64, 1, 20], 333), ([5, 5], 33001)])
def test_tokens_match(rows, V, with_probs, T):
    g = torch.Generator().manual_seed(hash((len(rows), V, with_probs)) % 1000)
    starts, logits, probs, ids, u, ul = _inputs(g, rows, V, T, with_probs)
    _run(logits, starts, ids, probs, u, ul, T, max(rows))
    _run(logits, starts, ids, probs, u, ul, T, min(64, max(rows) + 2), stride=3)


def test_all_accepted_and_all_refused():
    g = torch.Generator().manual_seed(5)
    starts, logits, probs, ids, u, ul = _inputs(g, [4, 4], 500, 1.0, True, noise=0.0)
    want = _run(logits, starts, ids, probs, u * 0.999, ul, 1.0, 4)     # q = p but for its rounding to 32 bits
    assert all(len(t) >= 1 for t in want)
    # drafts that the target gives no weight
    logits[torch.arange(8), ids.long()] = -math.inf
    want = _run(logits, starts, ids, probs, u, ul, 1.0, 4)
    assert [len(t) for t in want] == [1, 1]
    # and drafts that it gives all
    logits.fill_(-math.inf)
    logits[torch.arange(8), ids.long()] = 3.0
    for p in (probs, None):
        want = _run(logits, starts, ids, p, u, ul, 1.0, 4)
        assert [len(t) for t in want] == [4, 4]


@pytest.mark.parametrize("T", [0.0, 0.7])
def test_strange_rows(T):
    """Infinities, NaN, ties, rows with nothing, drafts outside the vocabulary."""
    g = torch.Generator().manual_seed(6)
    V = 5000
    rows = [3] * 12
    starts, logits, probs, ids, u, ul = _inputs(g, rows, V, 0.7, True)
    logits[0] = -math.inf                             # nothing at all
    logits[3] = math.nan
    logits[6, ::2] = math.nan                         # half the row
    logits[9, 4321] = math.inf                        # one takes all
    logits[12, 100] = logits[12, 4800] = math.inf     # two share
    logits[15] = 1.5                                  # all equal
    logits[18] = torch.finfo(torch.float32).min       # the lowest value everywhere
    logits[21, 7] = logits[21, 4999] = 50.0           # a tie at the top
    ids[24], ids[27] = -3, V                          # outside
    probs[30] = 0.0                                   # a draft that its model could not have drawn
    probs[33] = math.nan
    for p in (probs, None):
        _run(logits, starts, ids, p, u, ul, T, 3)


def test_ends_of_the_draw():
    """u_last at 0 and just below 1; a draw with weight in one id only."""
    g = torch.Generator().manual_seed(8)
    V = 9000
    starts, logits, probs, ids, u, ul = _inputs(g, [1] * 6, V, 1.0, False)
    ul = torch.tensor([0.0, 1 - 2.0 ** -24, 0.5, 0.0, 1 - 2.0 ** -24, 0.999])
    logits[0, :700] = -math.inf                       # the lowest id with weight
    logits[1, 4500:] = -math.inf                      # the highest
    logits[2:] = -math.inf
    for r, v in ((2, 0), (3, 8999), (4, 4096), (5, 1023)):
        logits[r, v] = -5.0
    want = _run(logits, starts, ids, None, u, ul, 1.0, 1)
    assert want[0] == [700] and want[2:] == [[0], [8999], [4096], [1023]]


def test_rows_past_the_bounds_are_cut():
    """row_start beyond n_rows, and sequences of more rows than max_rows."""
    import paper_2501_13111_amd as fp
    g = torch.Generator().manual_seed(9)
    starts, logits, probs, ids, u, ul = _inputs(g, [5, 2], 300, 0.0, False, noise=0.0)
    out, n = torch.zeros(2, 3, dtype=torch.int32).cuda(), torch.zeros(2, dtype=torch.int32).cuda()
    fp.verify_draft(logits.cuda(), torch.tensor([0, 5, 1000], dtype=torch.int32).cuda(), ids.cuda(), None, None, out, n,
                    temperature=0.0)
    best = logits.argmax(-1)
    assert n.tolist() == [3, 2] and out[0].tolist() == best[:3].tolist() and out[1].tolist() == best[5:7].tolist() + [-1]


@pytest.mark.parametrize("T", [0.0, 0.9])
@pytest.mark.parametrize("rows,V", [([3, 2], 2**20), ([2], 2**20 - 1), ([1, 0, 4] * 1365 + [2], 40)])
def test_largest_vocabulary_and_most_sequences(rows, V, T):
    g = torch.Generator().manual_seed(V % 977)
    starts, logits, probs, ids, u, ul = _inputs(g, rows, V, T, True)
    _run(logits, starts, ids, probs, u, ul, T, max(rows))


@pytest.mark.parametrize("T", [0.0, 0.9])
def test_captured_calls_and_another_stream(T):
    """Replays with other logits, drafts and row counts, eager calls between them."""
    import paper_2501_13111_amd as fp
    g = torch.Generator().manual_seed(21)
    B, R, V = 7, 5, 9000
    N = B * R
    logits, probs = torch.zeros(N, V, device="cuda"), torch.zeros(N, V, device="cuda")
    starts, ids = torch.zeros(B + 1, dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    u, ul = torch.zeros(N, device="cuda"), torch.zeros(B, device="cuda")
    outs = [(torch.empty(B, R, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")) for _ in range(3)]
    ws = [fp.verify_draft_workspace(N, V, B) for _ in range(2)]

    def run(o, w, stream=None):
        fp.verify_draft(logits, starts, ids, u, ul, *o, draft_probs=probs, temperature=T, workspace=w, stream=stream)

    run(outs[0], ws[0])
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        run(outs[0], ws[0])
    side = torch.cuda.Stream()
    for step in range(4):
        rows = torch.randint(0, R + 1, (B,), generator=g).tolist()
        st, lg, pr, dr, uu, uul = _inputs(g, rows, V, T or 1.0, True)
        n = st[-1]
        starts.copy_(torch.tensor(st, dtype=torch.int32))
        logits[:n], probs[:n], ids[:n], u[:n] = lg.cuda(), pr.cuda(), dr.cuda(), uu.cuda()
        ul.copy_(uul)
        torch.cuda.synchronize()
        gr.replay()
        with pytest.raises(ValueError):
            run(outs[1], None, stream=side)
        run(outs[1], ws[1], stream=side)
        torch.cuda.synchronize()
        run(outs[2], None)
        torch.cuda.synchronize()
        want = ref.verify(lg, st, dr, pr if T > 0 else None, uu, uul, T, R)
        for o, k in outs:
            assert [o[b, :k[b]].tolist() for b in range(B)] == want, step
