"""Binding of decoding with several continuations of a sequence on one paged cache (include/fp.h): drafted trees and
beams -- argument marshalling only, like ``paged``, whose rules for devices, streams and captured calls hold here too.
"""
from __future__ import annotations

import ctypes

import torch

from .binding import _check, load
from .paged import Chunk, PagedKV, _attn, _call, _PagedKv, _tensor, _workspace

MAX_ROWS = 1 << 24       # the most rows of a chunk


def attn_tree(kv: PagedKV, chunk: Chunk, parent, q, out, scale: float | None = None, workspace=None, stream=None):
    """``attn_chunk`` where the chunk's rows are nodes of drafted trees: row i of a sequence is the child of its row
    parent[row i] (int32 [rows]; -1, or anything that is no earlier row of the sequence: of none) and sees the context,
    its ancestors and itself.  Up to 64 rows a sequence; workspaces are those of ``attn_chunk_workspace``."""
    _attn("fp_attn_tree", (parent,), kv, chunk, q, out, scale, workspace, stream)


def _layers(kvs):
    """The C array of the layers' caches, and their device."""
    kvs = [kvs] if isinstance(kvs, PagedKV) else list(kvs)
    if not kvs:
        raise ValueError("no paged cache")
    if any(kv.device != kvs[0].device for kv in kvs):
        raise ValueError("the layers' pages must be on one device")
    return (_PagedKv * len(kvs))(*[kv.struct for kv in kvs]), kvs[0]


def kv_keep(kvs, chunk: Chunk, path, n_keep, stream=None):
    """In every cache of kvs (a PagedKV, or one per layer) node path[b, j] of sequence b moves to place j of its nodes,
    j < n_keep[b]: path int32 [sequences, any] and n_keep int32 [sequences], as ``verify_tree`` leaves them.  Before
    ctx_len grows by n_keep."""
    c, kv = _layers(kvs)
    B = chunk.n_seqs
    if not isinstance(path, torch.Tensor) or path.dim() != 2 or path.shape[0] != B:
        raise ValueError(f"path must be a [{B}, nodes] tensor")
    pp = _tensor(path, torch.int32, "path", device=kv.device)
    np_ = _tensor(n_keep, torch.int32, "n_keep", (B,), device=kv.device)
    if path.shape[1] == 0:
        return
    _call("fp_kv_keep", kv.device, stream, c, len(c), chunk.c(kv, MAX_ROWS), pp, path.shape[1], np_)


def verify_tree_workspace(n_rows: int, vocab: int, device="cuda"):
    """A workspace for verify_tree calls of up to n_rows rows.  Calls that may overlap (other streams, graphs
    replayed side by side) need one each."""
    n = ctypes.c_size_t()
    _check(load().fp_verify_tree_workspace(1, int(n_rows), int(vocab), ctypes.byref(n)), "fp_verify_tree_workspace")
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device=device)


def _logits(logits):
    """Address and row stride of float32 [rows, vocab] logits."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2:
        raise ValueError("logits must be a 2-dimensional tensor")
    N, V = logits.shape
    p = _tensor(logits, torch.float32, "logits", contiguous=False)
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("logits rows must be contiguous")
    return p or None, logits.stride(0) if N > 1 else V


def verify_tree(logits, row_start, parent, ids, u, out_ids, path, n_out, temperature: float = 1.0, workspace=None, stream=None):
    """Decide over drafted trees: logits float32 [rows, vocab], row_start int32 [sequences + 1], parent and ids
    int32 [rows] (node i's parent in its sequence and its token; node 0 is the root), u float32 [rows] in [0, 1) ->
    out_ids int32 [sequences, most rows of a sequence], the accepted tokens and the one drawn after them, path of that shape, the
    nodes they were drawn at (the root first), both -1 behind, and n_out int32 [sequences], their number.  u is not used at
    temperature 0 and may be None."""
    lp, ls = _logits(logits)
    if not isinstance(out_ids, torch.Tensor) or out_ids.dim() != 2:
        raise ValueError("out_ids must be a 2-dimensional tensor")
    (N, V), (B, R), dev = logits.shape, out_ids.shape, logits.device
    rp = _tensor(row_start, torch.int32, "row_start", (B + 1,), device=dev)
    pp = _tensor(parent, torch.int32, "parent", (N,), device=dev)
    ip = _tensor(ids, torch.int32, "ids", (N,), device=dev)
    up = _tensor(u, torch.float32, "u", (N,), device=dev) if u is not None else None
    op = _tensor(out_ids, torch.int32, "out_ids", device=dev)
    hp = _tensor(path, torch.int32, "path", (B, R), device=dev)
    np_ = _tensor(n_out, torch.int32, "n_out", (B,), device=dev)
    if workspace is None and stream is not None and stream != torch.cuda.current_stream(dev):
        raise ValueError("another stream than the current one needs a workspace of its own")
    w, wp, wn = _workspace(workspace, lambda: verify_tree_workspace(N, V, dev), dev)
    _call("fp_verify_tree", dev, stream, lp, ls, B, N, R, V, rp, pp, ip, up, float(temperature), op, hp, np_, wp, wn)


def beam_select_workspace(n_groups: int, n_beams: int, n_best: int, vocab: int, device="cuda"):
    """A workspace for beam_select calls of these sizes.  Calls that may overlap need one each."""
    n = ctypes.c_size_t()
    _check(load().fp_beam_select_workspace(int(n_groups), int(n_beams), int(n_best), int(vocab), ctypes.byref(n)),
           "fp_beam_select_workspace")
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device=device)


def beam_select(logits, scores, out_scores, out_parent, out_ids, done=None, out_done=None, eos_id: int = -1, pad_id: int = 0,
                workspace=None, stream=None):
    """The best continuations of every group's beams: logits float32 [groups * beams, vocab], scores float32 [groups, beams]
    (log probabilities so far), done None or bool [groups, beams] -> out_scores float32, out_parent (the beam within its group)
    and out_ids int32 and, if given, out_done bool, all [groups, best], best first; -inf, -1, -1 and False where there are
    fewer.  A done beam's one continuation is pad_id at its own score."""
    lp, ls = _logits(logits)
    if not isinstance(scores, torch.Tensor) or scores.dim() != 2 or not isinstance(out_ids, torch.Tensor) or out_ids.dim() != 2:
        raise ValueError("scores and out_ids must be 2-dimensional tensors")
    (N, V), (G, W), K, dev = logits.shape, scores.shape, out_ids.shape[1], logits.device
    if N != G * W:
        raise ValueError(f"{N} rows of logits for {G} groups of {W} beams")
    sp = _tensor(scores, torch.float32, "scores", device=dev)
    dp = _tensor(done, torch.bool, "done", (G, W), device=dev) if done is not None else None
    osp = _tensor(out_scores, torch.float32, "out_scores", (G, K), device=dev)
    opp = _tensor(out_parent, torch.int32, "out_parent", (G, K), device=dev)
    oip = _tensor(out_ids, torch.int32, "out_ids", (G, K), device=dev)
    odp = _tensor(out_done, torch.bool, "out_done", (G, K), device=dev) if out_done is not None else None
    if workspace is None and stream is not None and stream != torch.cuda.current_stream(dev):
        raise ValueError("another stream than the current one needs a workspace of its own")
    w, wp, wn = _workspace(workspace, lambda: beam_select_workspace(G, W, K, V, dev), dev)
    _call("fp_beam_select", dev, stream, lp, ls, G, W, K, V, sp, dp, int(eos_id), int(pad_id), osp, opp, oip, odp, wp, wn)


def beam_reorder(kvs, table, ctx_len, parent, table_out=None, stream=None):
    """Beam b of a group goes on from the caches (kvs: a PagedKV, or one per layer) of its beam parent[g, b]: table int32
    [groups * beams, pages], ctx_len int32 [groups * beams] (one length a group), parent int32 [groups, beams].  Full pages are
    shared by the rows of table_out (table itself if not given); a partly filled last page is copied into that of a beam which
    none goes on from."""
    c, kv = _layers(kvs)
    if not isinstance(parent, torch.Tensor) or parent.dim() != 2 or not isinstance(table, torch.Tensor) or table.dim() != 2:
        raise ValueError("parent and table must be 2-dimensional tensors")
    (G, W), width, dev = parent.shape, table.shape[1], kv.device
    pp = _tensor(parent, torch.int32, "parent", device=dev)
    tp = _tensor(table, torch.int32, "table", (G * W, width), device=dev)
    cp = _tensor(ctx_len, torch.int32, "ctx_len", (G * W,), device=dev)
    op = tp if table_out is None else _tensor(table_out, torch.int32, "table_out", (G * W, width), device=dev)
    _call("fp_beam_reorder", dev, stream, c, len(c), G, W, tp, width, width, cp, pp, op, width)
