// Device helpers of the paged-cache kernels: a chunk's sequences, sums and searches over them, and the
// pool's 32-position blocks.
#pragma once
#include "fp_device.h"

namespace fpk {

// A sequence of a chunk with the chunk's bounds enforced: whatever the device arrays hold, rows
// lie in [0, n_rows), new rows are at most max_new and positions end at max_len.
struct Seq {
    int row0, n, ctx, len;       // first row, rows, position of the first row, positions held
};
__device__ __forceinline__ Seq load_seq(const fp_chunk& c, int b) {
    const int r0 = min(max(c.row_start[b], 0), c.n_rows), r1 = min(max(c.row_start[b + 1], 0), c.n_rows);
    Seq s;
    s.row0 = r0;
    s.ctx = min(max(c.ctx_len[b], 0), c.max_len);
    s.n = min(min(max(r1 - r0, 0), c.max_new), c.max_len - s.ctx);
    s.len = s.ctx + s.n;
    return s;
}

// Inclusive sum over the wave's lanes, by data-parallel moves (a few cycles a step, where a shuffle
// through LDS takes a hundred): within rows of 16, then the rows' sums onwards.
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);      // row_shr:1, 2, 4, 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);      // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);      // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ int wave_total(int v) { return __builtin_amdgcn_readlane(wave_scan(v), 63); }

// Sequence l of a wave's lanes' sequences.
__device__ __forceinline__ Seq lane_seq(const Seq& s, int l) {
    return Seq{__builtin_amdgcn_readlane(s.row0, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.ctx, l),
               __builtin_amdgcn_readlane(s.len, l)};
}

// The last b < n (at most 4096) with before(b) <= u, or -1, for a before() that does not decrease: 64 of them at a time, so two
// loads after each other whatever n.  Where several sequences begin at one count, all but the last are empty.
template <class F>
__device__ __forceinline__ int last_at_most(int n, int u, F before) {
    const int lane = threadIdx.x & 63;
    int base = 0;
    if (n > 64) {
        const int b = 64 * lane;
        base = 64 * (__popcll(__ballot(b < n && before(b) <= u)) - 1);
        if (base < 0) return -1;
    }
    const int b = base + lane;
    return base + __popcll(__ballot(b < n && before(b) <= u)) - 1;
}

// The pool's block index of block blk (32 positions) of sequence b for kv head kvh: blocks of
// one (page, kv head) are consecutive.  -1 for a missing page.
__device__ __forceinline__ int pool_block(const fp_paged_kv& kv, const fp_chunk& c, int b, int kvh, int blk) {
    const int bpp = kv.page_size / VT_BLK;
    const int i = blk / bpp;
    const int page = i < c.table_stride ? c.table[(int64_t)b * c.table_stride + i] : -1;
    return page >= 0 && page < kv.n_pages ? (page * kv.n_kv_heads + kvh) * bpp + blk % bpp : -1;
}

}  // namespace fpk
