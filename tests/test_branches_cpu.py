"""Host-side tests of the entries for drafted trees and beams: arguments that they refuse before anything is launched,
sizes of their workspaces (no GPU needed), and the references that the GPU tests compare with."""
import ctypes
import math

import pytest
import torch

import branches_reference as bref
import paper_2501_13111_amd as fp
import test_paged_cpu as paged
from fpgen.workloads import Shape
from paper_2501_13111_amd import binding
from paper_2501_13111_amd.binding import Fingerprint
from paper_2501_13111_amd.paged import _PagedKv
from test_paged_cpu import CAPACITY, INVALID, UNSUPPORTED, P, chunk, kv


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _ref(x):
    return ctypes.byref(x) if x else None


def append(lib, pool, c, **kw):
    a = dict(parent=P, k=P, v=P, kv_stride=128, q=None, q_stride=0, n_heads=0, q_out=None, cos=None, sin=None, n_pos=0)
    a.update(kw)
    return lib.fp_kv_append_tree(_ref(pool), _ref(c), *a.values(), None)


def attn(lib, pool, c, **kw):
    a = dict(parent=P, q=P, q_stride=256, n_heads=4, scale=0.1, out=2 * P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_attn_tree(_ref(pool), _ref(c), *a.values(), None)


def keep(lib, pool, c, **kw):
    a = dict(n_layers=1, path=P, path_stride=4, n_keep=P)
    a.update(kw)
    return lib.fp_kv_keep(_ref(pool), a["n_layers"], _ref(c), a["path"], a["path_stride"], a["n_keep"], None)


@pytest.mark.parametrize("entry", [append, attn, keep])
@pytest.mark.parametrize("bad_kv,bad_chunk,code", [
    (dict(format=2), {}, INVALID), (dict(page_size=48), {}, INVALID), (dict(head_dim=96), {}, UNSUPPORTED), (dict(k=None), {}, INVALID),
    (dict(format=1, v_scales=P + 2), {}, INVALID), ({}, dict(n_seqs=4097), UNSUPPORTED), ({}, dict(max_new=0), INVALID),
    ({}, dict(max_len=129), CAPACITY), ({}, dict(row_start=None), INVALID), ({}, dict(table=None), INVALID),
    ({}, dict(max_new=65), UNSUPPORTED),
])
def test_caches_and_chunks_that_are_refused(lib, entry, bad_kv, bad_chunk, code):
    assert entry(lib, kv(**bad_kv), chunk(**bad_chunk)) == code
    assert lib.fp_last_error()
    assert entry(lib, None, chunk()) == INVALID and entry(lib, kv(), None) == INVALID


def test_trees_need_parents(lib):
    assert append(lib, kv(), chunk(), parent=None) == INVALID
    assert attn(lib, kv(), chunk(), parent=None) == INVALID
    # no rows: nothing to do, and nothing needed
    for entry in (append, attn):
        assert entry(lib, kv(), chunk(n_rows=0, max_new=64), parent=None) == 0
    assert keep(lib, kv(), chunk(n_rows=0)) == 0


@pytest.mark.parametrize("bad,code", [
    (dict(k=None), INVALID), (dict(kv_stride=120), INVALID), (dict(cos=P), INVALID), (dict(cos=P, sin=P, n_pos=127), CAPACITY),
    (dict(q=P, q_stride=256, n_heads=4, q_out=2 * P), INVALID),
    (dict(k=3 * P, v=3 * P, q=P, q_stride=256, n_heads=4, q_out=P + 512, cos=P, sin=P, n_pos=128), INVALID),
])
def test_tree_appends_that_are_refused(lib, bad, code):
    assert append(lib, kv(), chunk(), **bad) == code


@pytest.mark.parametrize("bad,code", [
    (dict(n_heads=5), INVALID), (dict(n_heads=34, q_stride=34 * 64), UNSUPPORTED), (dict(q=None), INVALID), (dict(out=P + 512), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(ws=None), INVALID), (dict(n=1024), CAPACITY),
])
def test_tree_attentions_that_are_refused(lib, bad, code):
    assert attn(lib, kv(), chunk(), **bad) == code


def test_keeps_that_are_refused(lib):
    for bad in (dict(n_layers=0), dict(n_layers=-1), dict(path=None), dict(n_keep=None), dict(path_stride=0)):
        assert keep(lib, kv(), chunk(), **bad) == INVALID
    for other in (dict(page_size=32), dict(n_kv_heads=1), dict(head_dim=128)):
        arr = (_PagedKv * 2)(kv(), kv(**other))
        assert lib.fp_kv_keep(arr, 2, _ref(chunk(max_len=64)), P, 4, P, None) == INVALID
    assert keep(lib, kv(n_kv_heads=200, n_pages=1), chunk(n_seqs=4096)) == UNSUPPORTED


S = Shape(2, 256, 4, 2, 64, 448, 4, 32, 100)


def test_tree_extends_that_are_refused(lib):
    def extend(h, kvs, c, parent=P, **kw):
        a = dict(x=P, y=2 * P, ws=P, n=1 << 40)
        a.update(kw)
        return lib.fp_extend_tree(h, (_PagedKv * len(kvs))(*kvs) if kvs else None, _ref(c), parent, *a.values(), None)
    with Fingerprint(S, unbacked=True) as f:
        ok, c = [kv(), kv(format=1)], chunk(max_len=100)
        assert extend(f._h, ok, c) == 0
        for kvs, ch, kw, code in [
            (None, c, {}, INVALID), (ok, None, {}, INVALID), ([kv(), kv(head_dim=128)], c, {}, INVALID),
            (ok, chunk(max_len=100, max_new=65), {}, UNSUPPORTED), (ok, chunk(max_len=101), {}, CAPACITY), (ok, c, dict(x=None), INVALID),
            (ok, c, dict(y=P + 512), INVALID), (ok, c, dict(ws=None), INVALID), (ok, c, dict(n=64), CAPACITY),
        ]:
            assert extend(f._h, kvs, ch, **kw) == code
    assert extend(None, ok, c) == INVALID


def verify(lib, **kw):
    a = dict(logits=P, stride=100, n_seqs=2, n_rows=6, max_rows=4, vocab=100, row_start=8 * P, parent=9 * P, ids=10 * P, u=11 * P, T=1.0,
             out=12 * P, path=13 * P, n_out=14 * P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_verify_tree(*a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(n_seqs=0), INVALID), (dict(n_seqs=4097), UNSUPPORTED), (dict(n_rows=-1), INVALID), (dict(n_rows=65536), UNSUPPORTED),
    (dict(vocab=0), INVALID), (dict(vocab=2**20 + 1, stride=2**21), UNSUPPORTED), (dict(max_rows=0), INVALID),
    (dict(max_rows=65), UNSUPPORTED), (dict(T=-1.0), INVALID), (dict(T=float("nan")), INVALID), (dict(T=float("inf")), INVALID),
    (dict(logits=None), INVALID), (dict(row_start=None), INVALID), (dict(parent=None), INVALID), (dict(ids=None), INVALID),
    (dict(out=None), INVALID), (dict(path=None), INVALID), (dict(n_out=None), INVALID), (dict(u=None), INVALID), (dict(stride=99), INVALID),
    (dict(ws=None), INVALID), (dict(ws=P + 4), INVALID), (dict(n=16), CAPACITY),
    (dict(out=10 * P), INVALID), (dict(path=9 * P + 20), INVALID), (dict(n_out=P + 4 * 599), INVALID), (dict(n_out=8 * P + 8), INVALID),
    (dict(path=12 * P + 28), INVALID), (dict(n_out=12 * P), INVALID), (dict(out=11 * P), INVALID),
])
def test_tree_verifications_that_are_refused(lib, bad, code):
    assert verify(lib, **bad) == code
    n = ctypes.c_size_t()
    if {"n_seqs", "n_rows", "vocab"} & set(bad):
        a = dict(n_seqs=2, n_rows=6, vocab=100)
        a.update({k: v for k, v in bad.items() if k in a})
        assert lib.fp_verify_tree_workspace(*a.values(), ctypes.byref(n)) == code
    assert lib.fp_verify_tree_workspace(2, 6, 100, None) == INVALID


def select(lib, **kw):
    a = dict(logits=P, stride=1000, groups=3, beams=4, best=8, vocab=1000, scores=8 * P, done=9 * P, eos=2, pad=0, os=10 * P, op=11 * P,
             oi=12 * P, od=13 * P, ws=P, n=1 << 40)
    a.update(kw)
    return lib.fp_beam_select(*a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(groups=0), INVALID), (dict(beams=0), INVALID), (dict(best=0), INVALID), (dict(vocab=0), INVALID), (dict(beams=65), UNSUPPORTED),
    (dict(best=65), UNSUPPORTED), (dict(vocab=2**20 + 1, stride=2**21), UNSUPPORTED), (dict(groups=1024, beams=64), UNSUPPORTED),
    (dict(groups=65536, beams=1), UNSUPPORTED), (dict(logits=None), INVALID), (dict(scores=None), INVALID), (dict(os=None), INVALID),
    (dict(op=None), INVALID), (dict(oi=None), INVALID), (dict(stride=999), INVALID), (dict(ws=None), INVALID), (dict(ws=P + 8), INVALID),
    (dict(n=256), CAPACITY), (dict(os=8 * P + 44), INVALID), (dict(oi=P + 4 * 11000), INVALID), (dict(od=9 * P + 11), INVALID),
    (dict(op=9 * P), INVALID), (dict(oi=10 * P + 92), INVALID), (dict(od=11 * P + 95), INVALID),
])
def test_selections_that_are_refused(lib, bad, code):
    assert select(lib, **bad) == code
    n = ctypes.c_size_t()
    if {"groups", "beams", "best", "vocab"} & set(bad):
        a = dict(groups=3, beams=4, best=8, vocab=1000)
        a.update({k: v for k, v in bad.items() if k in a})
        assert lib.fp_beam_select_workspace(*a.values(), ctypes.byref(n)) == code
    assert lib.fp_beam_select_workspace(3, 4, 8, 1000, None) == INVALID


def reorder(lib, pools=None, **kw):
    pools = pools or [kv()]
    a = dict(n_layers=len(pools), groups=2, beams=3, table=P, stride=5, width=4, ctx=2 * P, parent=3 * P, out=4 * P, out_stride=4)
    a.update(kw)
    return lib.fp_beam_reorder((_PagedKv * len(pools))(*pools), *a.values(), None)


@pytest.mark.parametrize("bad,code", [
    (dict(n_layers=0), INVALID), (dict(groups=0), INVALID), (dict(beams=0), INVALID), (dict(beams=65), UNSUPPORTED),
    (dict(groups=1024, beams=64), UNSUPPORTED), (dict(table=None), INVALID), (dict(ctx=None), INVALID), (dict(parent=None), INVALID),
    (dict(out=None), INVALID), (dict(width=0), INVALID), (dict(stride=3), INVALID), (dict(out_stride=3), INVALID),
    (dict(out=P), INVALID),                                     # the table, with other rows
    (dict(out=P + 8, out_stride=5), INVALID), (dict(out=2 * P + 20), INVALID), (dict(out=3 * P - 92), INVALID),
    (dict(pools=[kv(), kv(page_size=32)]), INVALID), (dict(pools=[kv(k=None)]), INVALID), (dict(pools=[kv(head_dim=80)]), UNSUPPORTED),
])
def test_reorderings_that_are_refused(lib, bad, code):
    assert reorder(lib, **bad) == code


def test_null_caches(lib):
    assert lib.fp_beam_reorder(None, 1, 2, 3, P, 4, 4, P, P, P, 4, None) == INVALID
    assert lib.fp_kv_keep(None, 1, _ref(chunk()), P, 4, P, None) == INVALID


def test_the_binding_refuses_host_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    m = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="HIP"):
        fp.verify_tree(torch.zeros(4, 8), i[:3], i, i, None, m, m, i[:2], temperature=0)
    with pytest.raises(ValueError):
        fp.verify_tree(torch.zeros(4), i[:3], i, i, None, m, m, i[:2], temperature=0)
    with pytest.raises(ValueError, match="HIP"):
        fp.beam_select(torch.zeros(4, 8), torch.zeros(2, 2), torch.zeros(2, 2), m, m)
    with pytest.raises(ValueError):
        fp.beam_select(torch.zeros(4, 8), torch.zeros(4), torch.zeros(2, 2), m, m)
    with pytest.raises(ValueError):
        fp.kv_keep([], None, m, i)
    with pytest.raises(ValueError):
        fp.beam_reorder([], m, i, m)


# ------------------------------------------------------------------ the references themselves
def test_lines_of_a_tree():
    assert bref.lines([-1, 0, 0, 1, 3, 9, 5]) == [[0], [0, 1], [0, 2], [0, 1, 3], [0, 1, 3, 4], [5], [5, 6]]


def test_beams_of_a_hand_made_group():
    """Two beams over three ids: log probabilities (ln .5, ln .3, ln .2) and (ln .8, ln .1, ln .1), scores -1 and -2."""
    z = torch.log(torch.tensor([[[0.5, 0.3, 0.2], [0.8, 0.1, 0.1]]]))
    got = bref.beam_select(z, torch.tensor([[-1.0, -2.0]]), None, 4, 1, 0)[0]
    want = [(-1 + math.log(0.5), 0, 0, False), (-1 + math.log(0.3), 0, 1, True), (-2 + math.log(0.8), 1, 0, False), (-1 + math.log(0.2), 0, 2, False)]
    assert [g[1:] for g in got] == [w[1:] for w in want]
    assert all(abs(g[0] - w[0]) < 1e-6 for g, w in zip(got, want))
    # the first beam finished: it stands for itself; a beam without a score has nothing
    got = bref.beam_select(z, torch.tensor([[-1.0, -math.inf]]), torch.tensor([[True, False]]), 2, 1, 7)[0]
    assert got == [(-1.0, 0, 7, True), (-math.inf, -1, -1, False)]


def test_reordering_by_hand():
    """Five positions in pages of two: beams 0, 1, 2 go on from 2, 2, 0; the last page of beam 1 is free."""
    new, copies = bref.reorder([[1, 2, 3, 4], [5, 6, 7, 8], [9, 10, 11, 12]], 5, [2, 2, 0], 2, 3)
    assert new == [[9, 10, 11, 4], [9, 10, 7, 8], [1, 2, 3, 12]] and copies == [(11, 7)]
    new, copies = bref.reorder([[1, 2, 3], [5, 6, 7]], 4, [1, 1], 2, 2)     # whole pages
    assert new == [[5, 6, 3], [5, 6, 7]] and copies == []


def test_walk_of_a_hand_made_tree():
    z = torch.full((4, 3), -5.0)
    z[0, 2] = z[2, 1] = z[1, 0] = z[3, 0] = 5.0
    assert bref.verify_tree(z, [0, 4], [-1, 0, 0, 2], [9, 1, 2, 1], None, 0.0, 8) == [([2, 1, 0], [0, 2, 3])]
    assert bref.verify_tree(z, [0, 4], [-1, 0, 0, 2], [9, 1, 1, 1], None, 0.0, 8) == [([2], [0])]
    assert paged.P == P
