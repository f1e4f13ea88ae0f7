"""Binding of the paged KV cache, the attention of a chunk over it and the verification of
drafted tokens (include/fp.h) -- argument marshalling only, like ``binding``.

Tensors must live on one HIP device; calls run on that device, on ``stream`` or that device's
current stream, and may be captured into a graph.
"""
from __future__ import annotations

import ctypes
import math

import torch

from .binding import KVQ, _check, load

VT_BLK = 32      # positions per transposed block of values
MAX_POSITIONS = 2**31 - 1024     # the largest max_len


class _PagedKv(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class _Chunk(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("max_new", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("row_start", ctypes.c_void_p),
                ("ctx_len", ctypes.c_void_p), ("table", ctypes.c_void_p)]


def _tensor(t, dtype, name, shape=None, contiguous=True, device=None):
    """t's address, after checking that it is a HIP tensor of that type (and shape, and device)."""
    try:
        if t.dtype is dtype and t.is_cuda and (shape is None or t.shape == shape) and \
                (device is None or t.device == device) and (not contiguous or t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor") from None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    raise ValueError(f"{name} must be contiguous")


_fn = {}
# the current stream's handle without a Stream object (about a microsecond less a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
# tensors on a device have initialised torch's side of it
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(name, device, stream, *args):
    """Run an entry point on `device`, on `stream` or the device's current stream."""
    f = _fn.get(name)
    if f is None:
        f = _fn[name] = getattr(load(), name)
    if stream is None:
        s = _raw_stream(device.index)
    else:
        if stream.device != device:
            raise ValueError(f"the stream is on {stream.device}, the tensors on {device}")
        s = stream.cuda_stream
    if _device() == device.index:
        rc = f(*args, s)
    else:
        with torch.cuda.device(device):
            rc = f(*args, s)
    if rc != 0:
        _check(rc, name)


class _Fixed:
    """Attributes that are set once: calls use the addresses and bounds taken from them when the object was
    made.  Contents of tensors may change in place."""

    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:
            raise AttributeError(f"{name} cannot be replaced, make a new {type(self).__name__}")
        self.__dict__[name] = value

    def __delattr__(self, name):
        raise AttributeError(f"{name} cannot be taken out of a {type(self).__name__}")


class PagedKV(_Fixed):
    """One layer's paged cache over the caller's pool tensors.

    k [n_pages, n_kv_heads, page_size, head_dim], v [n_pages, n_kv_heads, page_size / 32, head_dim,
    32], bfloat16 or int8; int8 also k_scales and v_scales, float16 [n_pages, n_kv_heads, page_size].
    ``PagedKV.empty`` allocates them.  Other tensors make another PagedKV.
    """

    def __init__(self, k, v, k_scales=None, v_scales=None):
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k must be a [pages, kv heads, page size, head_dim] tensor")
        n, h, ps, d = k.shape
        if k.dtype not in (torch.bfloat16, torch.int8):
            raise ValueError(f"k must be bfloat16 or int8, not {k.dtype}")
        self.kvq = "int8" if k.dtype == torch.int8 else "bf16"
        if ps % VT_BLK != 0 or ps == 0:
            raise ValueError(f"page size {ps} is not a positive multiple of {VT_BLK}")
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = n, h, ps, d
        self.device = k.device
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        kp = _tensor(k, k.dtype, "k")
        vp = _tensor(v, k.dtype, "v", (n, h, ps // VT_BLK, d, VT_BLK), device=k.device)
        sp = [None, None]
        if self.kvq == "int8":
            sp = [_tensor(t, torch.float16, nm, (n, h, ps), device=k.device)
                  for t, nm in ((k_scales, "k_scales"), (v_scales, "v_scales"))]
        elif k_scales is not None or v_scales is not None:
            raise ValueError("a bf16 cache has no scales")
        self.struct = _PagedKv(KVQ[self.kvq], n, ps, h, d, kp, vp, *sp)
        self.c = ctypes.byref(self.struct)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, kvq: str = "bf16", device="cuda"):
        """A cache of unwritten pages."""
        dt = {"bf16": torch.bfloat16, "int8": torch.int8}[kvq]
        k = torch.empty(n_pages, n_kv_heads, page_size, head_dim, dtype=dt, device=device)
        v = torch.empty(n_pages, n_kv_heads, page_size // VT_BLK, head_dim, VT_BLK, dtype=dt, device=device)
        sc = [torch.empty(n_pages, n_kv_heads, page_size, dtype=torch.float16, device=device) for _ in range(2)]
        return cls(k, v, *sc) if kvq == "int8" else cls(k, v)


class Chunk(_Fixed):
    """A ragged batch of rows: row_start int32 [n_seqs + 1], ctx_len int32 [n_seqs], table int32
    [n_seqs, pages per sequence] on the device, and host bounds on a sequence's rows (max_new) and
    on its positions with them (max_len; the table's whole width if not given).  The tensors' contents
    may change between calls; other tensors or bounds make another Chunk."""

    def __init__(self, row_start, ctx_len, table, max_new: int, max_len: int | None = None):
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table must be a [sequences, pages] tensor")
        B = table.shape[0]
        self.device = table.device
        self.row_start, self.ctx_len, self.table = row_start, ctx_len, table
        self.max_new, self.max_len = int(max_new), max_len if max_len is None else int(max_len)
        self.width = table.shape[1]
        self._p = (_tensor(row_start, torch.int32, "row_start", (B + 1,), device=table.device),
                   _tensor(ctx_len, torch.int32, "ctx_len", (B,), device=table.device), _tensor(table, torch.int32, "table"))
        self.n_seqs = B
        self._c = {}             # the last C structures, by row count and page size

    def c(self, kv: PagedKV, n_rows: int):
        """The C structure for n_rows rows over kv's pages."""
        if kv.device != self.device:
            raise ValueError(f"the chunk is on {self.device}, the cache on {kv.device}")
        key = (n_rows, kv.page_size)
        c = self._c.get(key)
        if c is None:
            if len(self._c) >= 32:
                self._c.clear()
            max_len = self.max_len if self.max_len is not None else min(self.width * kv.page_size, MAX_POSITIONS)
            c = self._c[key] = ctypes.byref(_Chunk(self.n_seqs, n_rows, self.max_new, max_len, self.width, *self._p))
        return c


def _heads(t, name, n_rows, head_dim, device):
    """Address and row stride of a bf16 [rows, heads, head_dim] tensor whose heads lie side by side
    (a view of a wider row included), and its head count."""
    p = _tensor(t, torch.bfloat16, name, contiguous=False, device=device)
    shape = t.shape
    if len(shape) != 3 or shape[2] != head_dim or (n_rows is not None and shape[0] != n_rows):
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [{n_rows if n_rows is not None else 'rows'}, heads, {head_dim}]")
    n, h, _ = shape
    if n * h == 0:
        return p or None, h * head_dim, h
    rs, hs, ds = t.stride()
    if ds != 1 or (h > 1 and hs != head_dim):
        raise ValueError(f"{name}'s heads must lie side by side")
    return p, rs if n > 1 else h * head_dim, h


def kv_append(kv: PagedKV, chunk: Chunk, k, v, q=None, q_out=None, cos=None, sin=None, stream=None, parent=None):
    """Write k and v (bf16 [rows, kv heads, head_dim], views of a fused projection included) to the
    chunk's positions.  With cos and sin (float32 [positions, head_dim / 2]) k is rotated first, and
    q, if given, into q_out.  With parent (int32 [rows]) the rows are nodes of drafted trees
    (``branches.attn_tree``), rotated by their depth."""
    N, d, dev = k.shape[0], kv.head_dim, kv.device
    kp, ks, kh = _heads(k, "k", N, d, dev)
    vp, vs, vh = _heads(v, "v", N, d, dev)
    if kh != kv.n_kv_heads or vh != kv.n_kv_heads:
        raise ValueError(f"k and v must have {kv.n_kv_heads} heads")
    if ks != vs:
        raise ValueError("k and v must have the same row stride")
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out come together")
    qp = op = None
    qs = H = 0
    if q is not None:
        qp, qs, H = _heads(q, "q", N, d, dev)
        op = _tensor(q_out, torch.bfloat16, "q_out", (N, H, d), device=dev)
    cp = sp = None
    n_pos = 0
    if cos is not None:
        n_pos = cos.shape[0]
        cp = _tensor(cos, torch.float32, "cos", (n_pos, d // 2), device=dev)
    if sin is not None:
        sp = _tensor(sin, torch.float32, "sin", (n_pos, d // 2), device=dev)
    if parent is not None:
        pp = _tensor(parent, torch.int32, "parent", (N,), device=dev)
    if N == 0:
        return
    if parent is not None:
        _call("fp_kv_append_tree", dev, stream, kv.c, chunk.c(kv, N), pp, kp, vp, ks, qp, qs, H, op, cp, sp, n_pos)
        return
    _call("fp_kv_append", dev, stream, kv.c, chunk.c(kv, N), kp, vp, ks, qp, qs, H, op,
          cp, sp, n_pos)


def kv_read(kv: PagedKV, chunk: Chunk, k_out, v_out, stream=None):
    """Read the chunk's positions back into k_out and v_out (bf16 [rows, kv heads, head_dim])."""
    shape = (k_out.shape[0], kv.n_kv_heads, kv.head_dim)
    kp = _tensor(k_out, torch.bfloat16, "k_out", shape, device=kv.device)
    vp = _tensor(v_out, torch.bfloat16, "v_out", shape, device=kv.device)
    if shape[0] == 0:
        return
    _call("fp_kv_read", kv.device, stream, kv.c, chunk.c(kv, shape[0]), kp, vp)


def attn_chunk_workspace(kv: PagedKV, chunk: Chunk, n_rows: int, n_heads: int):
    """A workspace for attn_chunk calls of these bounds.  Calls that may overlap (other streams,
    graphs replayed side by side) need one each."""
    n = ctypes.c_size_t()
    _check(load().fp_attn_chunk_workspace(kv.c, chunk.c(kv, n_rows), int(n_heads),
                                          ctypes.byref(n)), "fp_attn_chunk_workspace")
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device=kv.device)


def _workspace(workspace, make, device):
    w = make() if workspace is None else workspace
    return w, _tensor(w, torch.uint8, "workspace", device=device), w.numel()


def attn_chunk(kv: PagedKV, chunk: Chunk, q, out, scale: float | None = None, workspace=None, stream=None):
    """out [rows, heads, head_dim] = causal attention of the chunk's queries q (bf16, views of a
    fused projection included) over the cache, the chunk's own positions included.  scale defaults to
    1 / sqrt(head_dim); without a workspace the call takes one from torch's allocator, on the current
    stream, so it refuses another `stream` then."""
    _attn("fp_attn_chunk", (), kv, chunk, q, out, scale, workspace, stream)


def _attn(name, parent, kv, chunk, q, out, scale, workspace, stream):
    N = q.shape[0]
    qp, qs, H = _heads(q, "q", N, kv.head_dim, kv.device)
    op = _tensor(out, torch.bfloat16, "out", (N, H, kv.head_dim), device=kv.device)
    parent = tuple(_tensor(p, torch.int32, "parent", (N,), device=kv.device) for p in parent)
    if N == 0:
        return
    if workspace is None and stream is not None and stream != torch.cuda.current_stream(kv.device):
        raise ValueError("another stream than the current one needs a workspace of its own")
    w, wp, wn = _workspace(workspace, lambda: attn_chunk_workspace(kv, chunk, N, H), kv.device)
    _call(name, kv.device, stream, kv.c, chunk.c(kv, N), *parent, qp, qs, H,
          1.0 / math.sqrt(kv.head_dim) if scale is None else float(scale), op, wp, wn)


def verify_draft_workspace(n_rows: int, vocab: int, n_seqs: int | None = None, device="cuda"):
    """A workspace for verify_draft calls of up to n_rows rows (and n_seqs sequences, at most one a
    row if not given)."""
    n = ctypes.c_size_t()
    _check(load().fp_verify_draft_workspace(int(n_seqs if n_seqs is not None else max(1, min(n_rows, 4096))), int(n_rows),
                                            int(vocab), ctypes.byref(n)), "fp_verify_draft_workspace")
    return torch.empty(max(n.value, 16), dtype=torch.uint8, device=device)


def verify_draft(logits, row_start, draft_ids, u, u_last, out_ids, n_out, draft_probs=None, temperature: float = 1.0,
                 workspace=None, stream=None):
    """Decide over drafted tokens: logits float32 [rows, vocab], row_start int32 [sequences + 1],
    draft_ids int32 [rows], draft_probs None or float32 [rows, vocab], u float32 [rows] and u_last
    float32 [sequences] in [0, 1) -> out_ids int32 [sequences, most rows of a sequence] (-1 behind
    the last token) and n_out int32 [sequences].  u, u_last and draft_probs are not used at
    temperature 0 and may be None."""
    if not isinstance(logits, torch.Tensor) or logits.dim() != 2 or not isinstance(out_ids, torch.Tensor) or out_ids.dim() != 2:
        raise ValueError("logits and out_ids must be 2-dimensional tensors")
    (N, V), (B, R), dev = logits.shape, out_ids.shape, logits.device

    def rows(t, name):
        p = _tensor(t, torch.float32, name, (N, V), contiguous=False, device=dev)
        if V > 1 and t.stride(1) != 1:
            raise ValueError(f"{name} rows must be contiguous")
        return p or None, t.stride(0) if N > 1 else V

    lp, ls = rows(logits, "logits")
    pp, ps = rows(draft_probs, "draft_probs") if draft_probs is not None else (None, 0)
    rp = _tensor(row_start, torch.int32, "row_start", (B + 1,), device=dev)
    ip = _tensor(draft_ids, torch.int32, "draft_ids", (N,), device=dev)
    up = _tensor(u, torch.float32, "u", (N,), device=dev) if u is not None else None
    ulp = _tensor(u_last, torch.float32, "u_last", (B,), device=dev) if u_last is not None else None
    op = _tensor(out_ids, torch.int32, "out_ids", device=dev)
    np_ = _tensor(n_out, torch.int32, "n_out", (B,), device=dev)
    if workspace is None and stream is not None and stream != torch.cuda.current_stream(dev):
        raise ValueError("another stream than the current one needs a workspace of its own")
    w, wp, wn = _workspace(workspace, lambda: verify_draft_workspace(N, V, B, dev), dev)
    _call("fp_verify_draft", dev, stream, lp, ls, B, N, R, V, rp, ip, pp, ps, up, ulp, float(temperature), op, np_, wp, wn)
