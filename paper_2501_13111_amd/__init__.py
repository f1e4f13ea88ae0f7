"""MI355X (gfx950) fingerprint forward pass: HIP kernels behind a C ABI (include/fp.h)
and a thin ctypes binding.  See ``binding.Fingerprint``, and ``paged`` for the paged KV cache."""
from .binding import Fingerprint, FpShape, FpError, fill_normal, load, lib_path  # noqa: F401

# paged needs torch, the rest does not.  Where torch is installed it is imported here, before the HIP library: that
# library then uses the HIP runtime that torch brought, and the process has one.
try:
    from .paged import (Chunk, PagedKV, attn_chunk, attn_chunk_workspace, kv_append, kv_read,  # noqa: F401
                        verify_draft, verify_draft_workspace)
    from .branches import (attn_tree, beam_reorder, beam_select, beam_select_workspace, kv_keep,  # noqa: F401
                           verify_tree, verify_tree_workspace)
except ModuleNotFoundError as e:
    if e.name != "torch":
        raise
