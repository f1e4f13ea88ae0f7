"""Values and keys of the context that are not finite, in the attention of drafted trees: every node sees them."""
import math

import pytest
import torch

import branches_reference as bref
import paged_reference as ref
import test_gpu_paged as paged

pytestmark = pytest.mark.gpu

CASES = {
    # the context's last whole block odd and even, contexts that end at a block's border and inside of one
    "streamed-16": (1, 4, 64, 32, [(60, 4), (96, 3), (31, 4), (127, 2), (129, 1)], 0),
    "streamed-32": (2, 8, 128, 64, [(60, 4), (96, 3), (31, 4), (127, 2)], 0),
    "streamed-64": (2, 2, 64, 64, [(60, 30), (96, 30), (31, 29), (127, 8)], 64),
    "streamed-64-of-64-dims-split": (2, 4, 64, 32, [(1500, 12), (60, 16), (2077, 9), (801, 16)], 0),
    "tiles-of-32": (2, 4, 128, 32, [(60, 40), (96, 33), (31, 64), (127, 17)], 0),
    "wide-whole": (8, 8, 128, 32, [(31 + 44 * b, 16 - b % 3) for b in range(20)], 0),
    "wide-whole-two-tiles": (8, 8, 128, 32, [(300 - 5 * b, 32 - b % 2) for b in range(10)], 0),
    # pieces that begin at odd and at even blocks
    "wide-split": (2, 8, 128, 64, [(2100, 16), (1090, 14), (1700, 16), (2077, 13), (1120, 15), (60, 16), (0, 16)], 64),
    "wide-split-one": (1, 16, 128, 32, [(3233, 8)], 32),
    "tiles-of-256": (1, 8, 128, 32, [(60, 40), (96, 33), (31, 64), (127, 36), (900, 50)], 32),
    "tiles-of-256-of-64-dims": (2, 4, 64, 32, [(60, 40), (96, 33), (31, 64), (127, 36), (900, 50)], 32),
}


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("case", sorted(CASES))
def test_values_of_the_context_that_are_not_finite_reach_every_node(case, kvq):
    """An infinite or NaN value, an int8 scale that is not finite, or a NaN key at one position of every block of the context in turn:
    no output of a node after it is finite (of the value's dim alone, bf16), and no other changes a bit."""
    nkv, G, d, page, lens, loose = CASES[case]
    fp = paged._fp()
    g, pool, table = paged._case(lens, page, nkv, d, kvq, 27)
    paged._fill(pool, table, lens, g, upto=lambda c, n: c + n)
    parent = torch.tensor(sum([bref.random_tree(g, n) for _, n in lens], []), dtype=torch.int32).cuda()
    chunk, starts = paged._chunk(lens, table, loose=loose)
    q = torch.randn(starts[-1], nkv * G, d, generator=g).bfloat16().cuda()
    kv, clean, out = pool.device(), torch.empty_like(q), torch.empty_like(q)
    fp.attn_tree(kv, chunk, parent, q, clean)
    assert torch.isfinite(clean.float()).all()
    rows = torch.tensor(sum([[b] * n for b, (_, n) in enumerate(lens)], []))
    head, dim = nkv - 1, 3
    mine = torch.arange(nkv * G) // G == head
    slot = ref.SLOT
    for blk in range(max(c for c, _ in lens) // 32 + 1):
        pos = 32 * blk + 7 * blk % 32
        for what in ("inf", "nan", "key"):
            bad = math.inf if what == "inf" else math.nan
            # one element of each sequence whose context has this position
            hit = [b for b, (c, _) in enumerate(lens) if pos < c]
            if not hit:
                continue
            pg, off = table[hit, pos // page].long().cuda(), pos % page
            if kvq == "int8":
                t, at = (kv.k_scales if what == "key" else kv.v_scales), (pg, head, off)
            elif what == "key":
                t, at = kv.k, (pg, head, off, dim)
            else:
                t, at = kv.v, (pg, head, off // 32, dim, int(slot[off % 32]))
            was = t[at].clone()
            t[at] = bad
            fp.attn_tree(kv, chunk, parent, q, out)
            t[at] = was
            sees = torch.isin(rows, torch.tensor(hit))
            sick = (sees[:, None] & mine)[..., None].expand(out.shape).clone()
            if kvq == "bf16" and what != "key":
                sick &= torch.arange(d) == dim
            sick = sick.cuda()
            fine = torch.isfinite(out.float())
            wrong = (fine & sick).any(-1).any(-1).nonzero()[:, 0].tolist()
            assert not wrong, f"{what} at {pos}: finite outputs in rows {wrong[:8]} after contexts {[lens[int(rows[r])][0] for r in wrong[:8]]}"
            assert torch.equal(ref.bits(out)[~sick], ref.bits(clean)[~sick]), f"{what} at {pos}"
