"""Drafted trees of more sequences than a workgroup plans by itself, with contexts long enough to be split, in tiles of 128 rows
(the most sequences, int8: of 32)."""
import math

import pytest
import torch

import branches_reference as bref
import paged_reference as ref
import test_gpu_paged as paged

pytestmark = pytest.mark.gpu

HALF_BF16 = paged.HALF_BF16
LENS = {
    # a few long contexts among short ones; all long, so that nearly every tile is split; the most sequences, most of them without rows
    "few-long": [(3000 if b % 90 == 7 else b * 13 % 190, 16 - b % 3) for b in range(300)],
    "long": [(1100 + b * 37 % 900, 15 + b % 2) for b in range(300)],
    "most": [(1500 + b % 50 if b % 64 == 9 else 0, 16 if b % 64 == 9 else 0) for b in range(4096)],
}


@pytest.mark.parametrize("kvq", ["bf16", "int8"])
@pytest.mark.parametrize("case,checked", [("few-long", 300), ("long", 40), ("most", 4096)])
def test_many_sequences_in_split_tiles(case, checked, kvq):
    """Against the reference, twice with the same bits; the workspace is as large as asked for and not a byte behind it is written."""
    fp = paged._fp()
    lens, page, nkv, G, d = LENS[case], 64, 1, 8, 128
    kv, table, g = paged._fill_gpu(lens, page, nkv, d, kvq, 37)
    max_new = 16
    chunk, starts = paged._chunk(lens, table, max_new=max_new)
    N = starts[-1]
    tg = torch.Generator().manual_seed(6)
    parent = sum([bref.random_tree(tg, n) for _, n in lens if n], [])
    pp = torch.tensor(parent, dtype=torch.int32).cuda()
    q = torch.randn(N, nkv * G, d, generator=g, device="cuda").bfloat16()
    n = fp.attn_chunk_workspace(kv, chunk, N, nkv * G).numel()
    room = torch.full((n + 4096,), 0xAB, dtype=torch.uint8).cuda()
    out, again = (torch.full((N + 2, nkv * G, d), 7.0, dtype=torch.bfloat16).cuda() for _ in range(2))
    for o in (out, again):
        fp.attn_tree(kv, chunk, pp, q, o[:N], workspace=room[:n])
    assert (room[n:] == 0xAB).all() and (out[N:] == 7.0).all()
    assert torch.equal(ref.bits(out), ref.bits(again))
    slot, root = ref.SLOT.cuda(), math.sqrt(d)
    step = max(1, len(lens) // checked)
    for b in list(range(0, len(lens), step)) + [len(lens) - 1]:
        ctx, new = lens[b]
        if new == 0:
            continue
        m, r = ctx + new, starts[b]
        pos = torch.arange(m, device="cuda")
        pg, off = table[b].cuda().long()[pos // page], pos % page
        k, v = kv.k[pg, 0, off].double(), kv.v[pg, 0, off // 32, :, slot[off % 32]].double()
        if kvq == "int8":
            k, v = k * kv.k_scales[pg, 0, off].double()[:, None], v * kv.v_scales[pg, 0, off].double()[:, None]
        seen = torch.zeros(new, m, dtype=torch.bool)
        seen[:, :ctx] = True
        for i, line in enumerate(bref.lines(parent[r:r + new])):
            seen[i, ctx + torch.tensor(line)] = True
        qq = q[r:r + new].double().reshape(new * G, d)
        s = (qq @ k.t().contiguous() / root).masked_fill(~seen.cuda().repeat_interleave(G, 0), -math.inf)
        p = torch.softmax(s, -1)
        want, mag = p @ v, p @ v.abs()
        # the output's rounding, and probabilities' (bf16; int8 caches: keys, values and probabilities in fp16, 2^-11 each); scores of at
        # most some tens keep fp32's share below 1e-4
        low = 2.0 ** -11 * (2 + 2 * (qq.abs() @ k.abs().t().contiguous() / root).amax(-1, keepdim=True)) if kvq == "int8" else HALF_BF16
        tol = HALF_BF16 * want.abs() + (low + 1e-4) * mag * (1 + HALF_BF16) + 2.0 ** -25
        assert ((out[r:r + new].double().reshape(new * G, d) - want).abs() <= tol).all(), b
