"""MI355X (gfx950) fingerprint forward pass: HIP kernels behind a C ABI (include/fp.h)
and a thin ctypes binding.  See ``binding.Fingerprint``, and ``paged`` for the paged KV cache."""
from .binding import Fingerprint, FpShape, FpError, fill_normal, load, lib_path  # noqa: F401
from .paged import (Chunk, PagedKV, attn_chunk, attn_chunk_workspace, kv_append, kv_read,  # noqa: F401
                    verify_draft, verify_draft_workspace)
