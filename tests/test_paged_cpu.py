"""Host-side tests of the paged cache's and the draft verification's entries: arguments that they refuse
before anything is launched, and sizes of their workspaces (no GPU needed)."""
import ctypes

import pytest
import torch

import paper_2501_13111_amd as fp
from fpgen.workloads import Shape
from paper_2501_13111_amd import binding
from paper_2501_13111_amd.binding import Fingerprint
from paper_2501_13111_amd.paged import _Chunk, _PagedKv

INVALID, CAPACITY, UNSUPPORTED = (next(c for c, n in binding.STATUS.items() if n == f"FP_ERR_{x}")
                                  for x in ("INVALID_ARG", "CAPACITY", "UNSUPPORTED"))
P = 1 << 20          # a 16-byte aligned address that nothing here reads


def kv(**kw):
    a = dict(format=0, n_pages=10, page_size=64, n_kv_heads=2, head_dim=64, k=P, v=P, k_scales=P, v_scales=P)
    a.update(kw)
    return _PagedKv(**a)


def chunk(**kw):
    a = dict(n_seqs=2, n_rows=6, max_new=3, max_len=128, table_stride=2, row_start=P, ctx_len=P, table=P)
    a.update(kw)
    return _Chunk(**a)


def append(lib, pool, c, **kw):
    a = dict(k=P, v=P, kv_stride=128, q=None, q_stride=0, n_heads=0, q_out=None, cos=None, sin=None, n_pos=0)
    a.update(kw)
    return lib.fp_kv_append(ctypes.byref(pool) if pool else None, ctypes.byref(c) if c else None, *a.values(), None)


def read(lib, pool, c, **kw):
    a = dict(k=P, v=2 * P)
    a.update(kw)
    return lib.fp_kv_read(ctypes.byref(pool) if pool else None, ctypes.byref(c) if c else None, *a.values(), None)


def attn(lib, pool, c, **kw):
    a = dict(q=P, q_stride=256, n_heads=4, scale=0.1, out=2 * P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_attn_chunk(ctypes.byref(pool) if pool else None, ctypes.byref(c) if c else None, *a.values(), None)


@pytest.fixture(scope="module")
def lib():
    return binding.load()


@pytest.mark.parametrize("entry", [append, read, attn])
@pytest.mark.parametrize("bad,code", [
    (dict(format=2), INVALID), (dict(n_pages=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(page_size=0), INVALID),
    (dict(page_size=48), INVALID), (dict(page_size=-64), INVALID), (dict(page_size=65568), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(n_pages=2**29, n_kv_heads=2), UNSUPPORTED),
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(k=P + 8), INVALID), (dict(format=1, k_scales=None), INVALID),
    (dict(format=1, v_scales=P + 2), INVALID),
])
def test_pages_that_are_refused(lib, entry, bad, code):
    assert entry(lib, kv(**bad), chunk()) == code
    assert lib.fp_last_error()


@pytest.mark.parametrize("entry", [append, read, attn])
@pytest.mark.parametrize("bad,code", [
    (dict(n_seqs=0), INVALID), (dict(n_rows=-1), INVALID), (dict(max_new=0), INVALID), (dict(max_len=0), INVALID),
    (dict(table_stride=0), INVALID), (dict(n_seqs=4097), UNSUPPORTED), (dict(n_rows=2**24 + 1), UNSUPPORTED),
    (dict(max_len=129), CAPACITY), (dict(max_len=2**31 - 1, table_stride=2**24), CAPACITY),
    (dict(row_start=None), INVALID), (dict(ctx_len=None), INVALID), (dict(table=None), INVALID),
])
def test_chunks_that_are_refused(lib, entry, bad, code):
    assert entry(lib, kv(), chunk(**bad)) == code


@pytest.mark.parametrize("entry", [append, read, attn])
def test_null_structures(lib, entry):
    assert entry(lib, None, chunk()) == INVALID
    assert entry(lib, kv(), None) == INVALID


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), INVALID), (dict(v=P + 2), INVALID), (dict(kv_stride=120), INVALID), (dict(kv_stride=132), INVALID),
    (dict(kv_stride=2**32 + 8), UNSUPPORTED),
    (dict(cos=P), INVALID), (dict(sin=P, n_pos=128), INVALID), (dict(cos=P + 4, sin=P, n_pos=128), INVALID),
    (dict(cos=P, sin=P, n_pos=127), CAPACITY),
    (dict(q=P, q_stride=256, n_heads=4, q_out=2 * P), INVALID),                      # queries without tables
    (dict(q=P, q_stride=256, n_heads=3, q_out=2 * P, cos=P, sin=P, n_pos=128), INVALID),
    (dict(q=P, q_stride=64 * 34, n_heads=34, q_out=2 * P, cos=P, sin=P, n_pos=128), UNSUPPORTED),
    (dict(q=P, q_stride=248, n_heads=4, q_out=2 * P, cos=P, sin=P, n_pos=128), INVALID),
    (dict(q=P, q_stride=256, n_heads=4, q_out=None, cos=P, sin=P, n_pos=128), INVALID),
    (dict(q=None, q_stride=256, n_heads=4, q_out=P, cos=P, sin=P, n_pos=128), INVALID),
    (dict(k=3 * P, v=3 * P, q=P, q_stride=256, n_heads=4, q_out=P + 512, cos=P, sin=P, n_pos=128), INVALID),      # over q
    (dict(k=P, v=3 * P, q=2 * P, q_stride=256, n_heads=4, q_out=P + 512, cos=P, sin=P, n_pos=128), INVALID),      # over k
])
def test_appends_that_are_refused(lib, bad, code):
    assert append(lib, kv(), chunk(), **bad) == code


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=P + 8), dict(v=P + 1024), dict(v=P)])
def test_reads_that_are_refused(lib, bad):
    assert read(lib, kv(), chunk(), **bad) == INVALID


@pytest.mark.parametrize("bad,code", [
    (dict(n_heads=0), INVALID), (dict(n_heads=5), INVALID), (dict(n_heads=34, q_stride=34 * 64), UNSUPPORTED), (dict(q=None), INVALID),
    (dict(out=None), INVALID), (dict(q=P + 2), INVALID), (dict(out=2 * P + 8), INVALID), (dict(q_stride=255), INVALID),
    (dict(q_stride=264 - 16), INVALID), (dict(out=P + 512), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID), (dict(n=1024), CAPACITY),
])
def test_attentions_that_are_refused(lib, bad, code):
    assert attn(lib, kv(), chunk(), **bad) == code


def test_no_rows_is_nothing_to_do(lib):
    assert append(lib, kv(), chunk(n_rows=0)) == 0
    assert read(lib, kv(), chunk(n_rows=0)) == 0
    assert attn(lib, kv(), chunk(n_rows=0)) == 0


def test_attention_workspace(lib):
    def need(k, c, H):
        n = ctypes.c_size_t()
        return lib.fp_attn_chunk_workspace(ctypes.byref(k), ctypes.byref(c), H, ctypes.byref(n)), n.value
    # no pointers needed; at most 64 MiB whatever the lengths; exactly enough is accepted (no rows: nothing runs)
    for c in (chunk(), chunk(n_rows=2**24, max_new=2**24, max_len=2**26, table_stride=2**20, n_seqs=4096)):
        rc, n = need(kv(k=None, v=None), c, 32)
        assert rc == 0 and 0 < n <= 80 << 20
    rc, n = need(kv(), chunk(n_rows=0), 4)
    assert attn(lib, kv(), chunk(n_rows=0), n=n) == 0 and attn(lib, kv(), chunk(n_rows=0), n=n - 1) == CAPACITY
    assert need(kv(), chunk(), 5)[0] == INVALID
    assert lib.fp_attn_chunk_workspace(ctypes.byref(kv()), ctypes.byref(chunk()), 4, None) == INVALID


@pytest.mark.parametrize("d,fmt", [(64, 0), (64, 1), (128, 0), (128, 1)])
def test_a_workspace_serves_smaller_calls(lib, d, fmt):
    n = ctypes.c_size_t()
    sizes = []
    for rows, new, length, seqs in [(1, 1, 32, 1), (4, 4, 500, 1), (40, 5, 2000, 8), (100, 9, 2000, 16), (500, 500, 4000, 16),
                                    (40000, 4000, 100000, 64), (40000, 4000, 100000, 65), (2**20, 2**20, 2**22, 4096)]:
        c = chunk(n_rows=rows, max_new=new, max_len=length, n_seqs=seqs, table_stride=2**17)
        k = kv(format=fmt, head_dim=d)
        assert lib.fp_attn_chunk_workspace(ctypes.byref(k), ctypes.byref(c), 16, ctypes.byref(n)) == 0
        sizes.append(n.value)
    assert sizes == sorted(sizes)


def verify(lib, **kw):
    a = dict(logits=P, stride=100, n_seqs=2, n_rows=6, max_rows=4, vocab=100, row_start=P, ids=P, probs=P, pstride=100, u=P, ul=P,
             T=1.0, out=P, n_out=P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_verify_draft(*a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(n_seqs=0), INVALID), (dict(n_seqs=4097), UNSUPPORTED), (dict(n_rows=-1), INVALID), (dict(n_rows=65536), UNSUPPORTED),
    (dict(vocab=0), INVALID), (dict(vocab=2**20 + 1, stride=2**21), UNSUPPORTED), (dict(max_rows=0), INVALID),
    (dict(max_rows=65), UNSUPPORTED), (dict(T=-1.0), INVALID), (dict(T=float("nan")), INVALID), (dict(T=float("inf")), INVALID),
    (dict(logits=None), INVALID), (dict(row_start=None), INVALID), (dict(ids=None), INVALID), (dict(out=None), INVALID),
    (dict(n_out=None), INVALID), (dict(u=None), INVALID), (dict(ul=None), INVALID), (dict(stride=99), INVALID),
    (dict(pstride=99), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID), (dict(n=16), CAPACITY),
])
def test_verifications_that_are_refused(lib, bad, code):
    assert verify(lib, **bad) == code
    n = ctypes.c_size_t()
    if {"n_seqs", "n_rows", "vocab"} & set(bad):
        a = dict(n_seqs=2, n_rows=6, vocab=100)
        a.update({k: v for k, v in bad.items() if k in a})
        assert lib.fp_verify_draft_workspace(*a.values(), ctypes.byref(n)) == code
    assert lib.fp_verify_draft_workspace(2, 6, 100, None) == INVALID


# ------------------------------------------------------------------ the layer stack
S = Shape(2, 256, 4, 2, 64, 448, 4, 32, 100)


def extend(lib, h, kvs, c, **kw):
    a = dict(x=P, y=2 * P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_extend(h, (_PagedKv * len(kvs))(*kvs) if kvs else None, ctypes.byref(c) if c else None, *a.values(), None)


def test_extends_that_are_refused(lib):
    with Fingerprint(S, unbacked=True) as f:
        ok, c = [kv(), kv(format=1)], chunk(max_len=100)
        assert extend(lib, f._h, ok, c) == 0                    # no storage: checked, nothing launched
        assert extend(lib, f._h, [kv(k=None, v=None)] * 2, c) == 0
        for kvs, ch, kw, code in [
            (None, c, {}, INVALID), (ok, None, {}, INVALID),
            ([kv(), kv(head_dim=128)], c, {}, INVALID), ([kv(), kv(n_kv_heads=4)], c, {}, INVALID),
            ([kv(), kv(page_size=40)], c, {}, INVALID), ([kv(), kv(page_size=32)], c, {}, CAPACITY),
            (ok, chunk(max_len=101), {}, CAPACITY), (ok, chunk(max_len=100, n_rows=129), {}, CAPACITY),
            (ok, c, dict(x=None), INVALID), (ok, c, dict(y=None), INVALID), (ok, c, dict(y=P + 512), INVALID),
            (ok, c, dict(ws=None), INVALID), (ok, c, dict(ws=P + 8), INVALID), (ok, c, dict(n=64), CAPACITY),
        ]:
            assert extend(lib, f._h, kvs, ch, **kw) == code, (kw, lib.fp_last_error())
        n = ctypes.c_size_t()
        arr = (_PagedKv * 2)(*ok)
        assert lib.fp_extend_workspace(f._h, arr, ctypes.byref(c), ctypes.byref(n)) == 0 and n.value > 0
        assert extend(lib, f._h, ok, c, n=n.value) == 0 and extend(lib, f._h, ok, c, n=n.value - 1) == CAPACITY
        assert lib.fp_extend_workspace(f._h, arr, ctypes.byref(c), None) == INVALID
    # caches of both formats: the largest layer's, whichever comes first
    with Fingerprint(Shape(2, 256, 4, 2, 64, 448, 4, 4096, 60000), unbacked=True) as f:
        c = chunk(n_rows=16000, max_new=8000, max_len=60000, table_stride=1000)
        sizes = {}
        for fmts in ((0, 0), (1, 1), (0, 1), (1, 0)):
            arr = (_PagedKv * 2)(*[kv(format=x) for x in fmts])
            assert lib.fp_extend_workspace(f._h, arr, ctypes.byref(c), ctypes.byref(n)) == 0
            sizes[fmts] = n.value
        assert sizes[1, 1] != sizes[0, 0] and sizes[0, 1] == sizes[1, 0] == max(sizes.values())
    assert extend(lib, None, ok, c) == INVALID


# ------------------------------------------------------------------ the binding
def test_the_binding_refuses_host_tensors():
    k = torch.zeros(4, 2, 32, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="HIP"):
        fp.PagedKV(k, torch.zeros(4, 2, 1, 64, 32, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        fp.PagedKV(k[0], k)
    with pytest.raises(ValueError):
        fp.PagedKV(k.float(), k)
    with pytest.raises(ValueError):
        fp.PagedKV(k[:, :, :31], k)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="HIP"):
        fp.Chunk(i, i[:2], torch.zeros(2, 4, dtype=torch.int32), max_new=1)
    with pytest.raises(ValueError):
        fp.Chunk(i, i[:2], i, max_new=1)
    with pytest.raises(ValueError):
        fp.verify_draft(torch.zeros(3), i, i, None, None, torch.zeros(1, 2, dtype=torch.int32), i, temperature=0)
