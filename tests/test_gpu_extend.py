"""The layer stack over ragged chunks on paged caches (fp_extend) against the oracle: prompts in
pieces, next tokens and both in one call, and a run of append, attention, LM head and draft
verification as speculative decoding uses them."""
import numpy as np
import pytest
import torch

import paged_reference as ref
from fpgen.workloads import Shape
from oracle.layer import Fingerprint as OracleFingerprint
from oracle.numerics import bf16_round
from tests.gpu_harness import TOL, bf16_to_np, np_to_bf16, rel_inf

pytestmark = pytest.mark.gpu


class Paged:
    """A fingerprint's caches and the sequences' tables."""

    def __init__(self, f, kvq, page, lens, seed=0):
        import paper_2501_13111_amd as fp
        s = f.shape
        need = [-(-n // page) for n in lens]
        g = torch.Generator().manual_seed(seed)
        self.table = ref.tables(g, need, sum(need) + 1, max(need)).cuda()
        self.kvs = [fp.PagedKV.empty(sum(need) + 1, page, s.n_kv_heads, s.head_dim, kvq) for _ in range(s.n_layers)]
        self.f, self.pos, self.max_len = f, [0] * len(lens), max(lens)

    def extend(self, xs, extra=0, graph=None):
        """xs: per sequence float32 rows [n, H] (n may be 0) -> per sequence outputs."""
        import paper_2501_13111_amd as fp
        H = self.f.shape.hidden
        starts = np.cumsum([0] + [len(x) for x in xs]).tolist()
        chunk = fp.Chunk(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(self.pos, dtype=torch.int32).cuda(),
                         self.table, max_new=max(1, max(len(x) for x in xs)), max_len=self.max_len)
        rows = np.concatenate([np.asarray(x, np.float32).reshape(-1, H) for x in xs] + [np.zeros((extra, H), np.float32)])
        x, y = np_to_bf16(rows), torch.empty(len(rows), H, dtype=torch.bfloat16, device="cuda")
        self.f.extend(self.kvs, chunk, x, y)
        self.pos = [p + len(v) for p, v in zip(self.pos, xs)]
        out = bf16_to_np(y)
        return [out[a:b] for a, b in zip(starts, starts[1:])]


CASES = [
    ("bf16-bf16", Shape(2, 256, 4, 4, 64, 688, 4, 64, 200), "bf16", "bf16", 32),
    ("int8-int8", Shape(2, 512, 8, 2, 64, 768, 3, 96, 160), "int8", "int8", 64),
    ("int4-bf16-gqa5", Shape(1, 640, 5, 1, 128, 768, 5, 40, 150), "int4", "bf16", 96),
    ("sp24-int8", Shape(1, 256, 4, 2, 64, 448, 2, 128, 140), "sp24", "int8", 32),
    ("wide-bf16", Shape(1, 2048, 16, 16, 128, 2752, 8, 64, 300), "bf16", "bf16", 128),
]


@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_chunks_match_the_oracle(case):
    """Sequences of different lengths, taken in pieces of one to many tokens, some of them idle in a call:
    every row's output is the oracle's for the whole sequence."""
    from paper_2501_13111_amd import Fingerprint
    _, s, wq, kvq, page = case
    rng = np.random.default_rng(3)
    plan = [[37, 5, 70], [1, 5, 0], [1, 1, 1], [0, 60, 2], [9, 1, 33]]
    lens = [sum(p[b] for p in plan) for b in range(3)]
    xs = [bf16_round(rng.normal(0, 1, (n, s.hidden)).astype(np.float32)) for n in lens]
    want = []
    for x in xs:
        want.append(OracleFingerprint(s, wq, kvq, seed=4).prefill(x[None])[0])
    with Fingerprint(s, wq, kvq, seed=4) as f:
        p = Paged(f, kvq, page, lens)
        at, errs = [0, 0, 0], []
        for step in plan:
            outs = p.extend([xs[b][at[b]:at[b] + step[b]] for b in range(3)], extra=2)
            for b in range(3):
                if step[b]:
                    errs.append(rel_inf(outs[b], want[b][at[b]:at[b] + step[b]]))
                at[b] += step[b]
    assert max(errs) <= TOL, errs


def test_the_handle_keeps_its_own_cache():
    """Steps of the handle's own sequences before and after an extend are the same bits."""
    from paper_2501_13111_amd import Fingerprint
    s = Shape(2, 256, 4, 2, 64, 448, 2, 32, 60)
    rng = np.random.default_rng(5)
    with Fingerprint(s, "int8", "int8", seed=6) as f:
        x = np_to_bf16(rng.normal(0, 1, (2 * 20, s.hidden)).astype(np.float32))
        y, u = torch.empty_like(x), torch.empty(2, s.hidden, dtype=torch.bfloat16, device="cuda")

        def run(between):
            f.prefill(x, y, 2, 20)
            t, outs = y.view(2, 20, -1)[:, -1].contiguous(), []
            for _ in range(3):
                between()
                f.decode_step(t, u)
                outs.append(u.clone())
                t.copy_(u)
            return outs
        plain = run(lambda: None)
        p = Paged(f, "bf16", 32, [60, 60])
        mixed = run(lambda: p.extend([rng.normal(0, 1, (n, s.hidden)).astype(np.float32) for n in (1, 17)]))
        assert f.position() == (23, 2)
    assert all(torch.equal(a, b) for a, b in zip(plain, mixed))


@pytest.mark.parametrize("rows", [1, 6])
def test_captured_extend(rows):
    """A step of every sequence captured once and replayed as the contexts grow."""
    import paper_2501_13111_amd as fp
    from paper_2501_13111_amd import Fingerprint
    s = Shape(2, 256, 4, 2, 64, 448, 6, 16, 120)
    g = torch.Generator().manual_seed(7)
    with Fingerprint(s, "bf16", "bf16", seed=8) as f:
        ps = [Paged(f, "int8", 32, [110] * rows) for _ in range(2)]
        for p in ps:
            for kv in p.kvs:
                for t in (kv.k, kv.v, kv.k_scales, kv.v_scales):
                    t.zero_()
        cl = torch.zeros(rows, dtype=torch.int32, device="cuda")
        rs = torch.arange(rows + 1, dtype=torch.int32).cuda()
        x = torch.empty(rows, s.hidden, dtype=torch.bfloat16, device="cuda")
        ys = [torch.empty_like(x) for _ in range(2)]
        chunks = [fp.Chunk(rs, cl, p.table, max_new=1, max_len=110) for p in ps]
        ws = [f.extend_workspace(p.kvs, c, rows) for p, c in zip(ps, chunks)]
        f.extend(ps[0].kvs, chunks[0], x, ys[0], workspace=ws[0])
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f.extend(ps[0].kvs, chunks[0], x, ys[0], workspace=ws[0])
        for i in range(8):
            x.copy_(torch.randn(x.shape, generator=g).bfloat16())
            cl.fill_(i)
            gr.replay()
            f.extend(ps[1].kvs, chunks[1], x, ys[1], workspace=ws[1])
            torch.cuda.synchronize()
            assert torch.equal(ys[0], ys[1]), i
            assert torch.isfinite(ys[0].float()).all()


@pytest.mark.parametrize("T", [0.0, 0.8])
def test_speculative_decoding_run(T):
    """Drafts of several sequences: embedding, layers over the pages, LM head of every new row, decision, and
    on from the accepted length (the refused tokens' positions are written again).  Logits are the oracle's for
    the accepted history, tokens the reference's decision on those logits."""
    import paper_2501_13111_amd as fp
    from paper_2501_13111_amd import Fingerprint
    s = Shape(2, 256, 4, 2, 64, 448, 16, 16, 96, vocab=512)
    B, K = 3, 4
    g = torch.Generator().manual_seed(9)
    with Fingerprint(s, "int8", "int8", seed=10) as f:
        p = Paged(f, "int8", 32, [90] * B)
        hist = [torch.randint(s.vocab, (n,), generator=g).tolist() for n in (7, 12, 3)]
        orc = OracleFingerprint(s, "int8", "int8", seed=10)

        def step(new):
            """new: per sequence tokens -> logits of their rows."""
            ids = torch.tensor(sum(new, []), dtype=torch.int32).cuda()
            x = torch.empty(len(ids), s.hidden, dtype=torch.bfloat16, device="cuda")
            f.embed(ids, x)
            starts = np.cumsum([0] + [len(t) for t in new]).tolist()
            chunk = fp.Chunk(torch.tensor(starts, dtype=torch.int32).cuda(), torch.tensor(p.pos, dtype=torch.int32).cuda(),
                             p.table, max_new=max(len(t) for t in new), max_len=90)
            y, lg = torch.empty_like(x), torch.empty(len(ids), s.vocab, device="cuda")
            f.extend(p.kvs, chunk, x, y)
            nxt = torch.empty(len(ids), dtype=torch.int32, device="cuda")
            for a in range(0, len(ids), s.max_batch):
                b = min(a + s.max_batch, len(ids))
                f.head(y[a:b], b - a, 1, nxt[a:b], lg[a:b])
            return starts, lg

        first = [h[:-1] for h in hist]
        step(first)
        p.pos = [len(t) for t in first]
        accepted = 0
        for it in range(4):
            # drafts: sometimes what the oracle would say, sometimes anything
            drafts = []
            for b in range(B):
                h, d = list(hist[b]), []
                for _ in range(K):
                    if torch.rand(1, generator=g) < 0.7:
                        y = orc.prefill(orc.embed(np.array(h))[None])
                        t = int(orc.head(y[:, -1])[1][0])
                    else:
                        t = int(torch.randint(s.vocab, (1,), generator=g))
                    d.append(t)
                    h.append(t)
                drafts.append(d)
            starts, lg = step([[hist[b][-1]] + drafts[b] for b in range(B)])
            for b in range(B):
                y = orc.prefill(orc.embed(np.array(hist[b] + drafts[b]))[None])
                want = orc.head(y[0, len(hist[b]) - 1:])[0]
                assert rel_inf(lg[starts[b]:starts[b + 1]].cpu().numpy(), want) <= TOL
            ids = torch.tensor(sum([d + [-1] for d in drafts], []), dtype=torch.int32)
            u, ul = torch.rand(len(ids), generator=g), torch.rand(B, generator=g)
            out, n = torch.empty(B, K + 1, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
            fp.verify_draft(lg, torch.tensor(starts, dtype=torch.int32).cuda(), ids.cuda(), u.cuda(), ul.cuda(), out, n, temperature=T)
            toks = ref.verify(lg.cpu(), starts, ids, None, u, ul, T, K + 1)
            assert [out[b, :n[b]].tolist() for b in range(B)] == toks
            for b in range(B):
                p.pos[b] += len(toks[b])
                hist[b] += toks[b]
                accepted += len(toks[b]) - 1
        assert accepted > 0 or T > 0        # (at T the nearly flat logits accept one token in hundreds)


@pytest.mark.parametrize("max_batch", [1, 3])
@pytest.mark.parametrize("wq,kvq", [("bf16", "int8"), ("int8", "bf16"), ("int4", "int8"), ("sp24", "bf16")])
def test_one_sequence_token_by_token(wq, kvq, max_batch):
    """A prompt, then calls of a single row."""
    from paper_2501_13111_amd import Fingerprint
    s = Shape(2, 256, 4, 2, 64, 512, max_batch, 40, 90)
    x = bf16_round(np.random.default_rng(11).normal(0, 1, (46, s.hidden)).astype(np.float32))
    want = OracleFingerprint(s, wq, kvq, seed=12).prefill(x[None])[0]
    with Fingerprint(s, wq, kvq, seed=12) as f:
        p = Paged(f, kvq, 32, [90])
        got = [p.extend([x[:40]])[0]] + [p.extend([x[i:i + 1]])[0] for i in range(40, 46)]
    assert rel_inf(np.concatenate(got), want) <= TOL
