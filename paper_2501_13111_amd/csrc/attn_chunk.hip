// Attention of a chunk of new tokens over a paged cache:
//     out[r, h] = sum_j softmax_j(scale q[r, h] . k_j) v_j,   j = 0 .. position of row r.
//
// The query heads of a group share a kv head's keys, so the rows that one pass over the keys
// serves are the pairs rho = (token) G + (head of the group) of a sequence, in tiles of 16 NT rows:
// any G fills the tiles, and row rho sees the positions up to ctx + rho / G.  Products in the
// transposed form on MFMA 16x16x32 (bf16; int8 codes are exact in bf16):
//     S^T = K Q^T     A = 16 keys, B = the tile's rows (columns)
//     O^T += V^T P^T  A = 16 dims of a value block, B = the probabilities
// so a lane holds the scores of 4 + 4 keys of a block for one row, and these are what it supplies
// to the second product (vt_slot order).  int8: a key's scale multiplies its scores, a value's its
// probabilities.  Online softmax per row in fp32, base 2.
//
// Work is split over the keys: from the lengths in device memory every workgroup works out the
// same plan, the 32-key blocks per piece Q = max(min_blocks, total blocks / target).  A piece is
// (sequence, kv head, row tile, Q consecutive blocks at most); its four waves take every fourth
// block and merge in LDS.  A tile of one piece is written out at once; the pieces of the others
// go to the workspace as unnormalised (o, m, l) and a second kernel joins them in order:
//     m = max m_i,  l = sum l_i 2^(m_i - m),  o = sum o_i 2^(m_i - m) / l.
// The plan depends on the inputs alone, so results repeat bit for bit.
#include <climits>

#include "attn_stream.h"

namespace fpk {

namespace {

template <int D, bool KV8, int NT>
__global__ void __launch_bounds__(256, NT == 1 ? 3 : NT == 4 && D == 128 ? 1 : 2) attn_chunk_kernel(AttnChunkArgs a) {
    __shared__ StreamLds<D, NT> lds;
    Unit un;
    if (!find_unit<16 * NT, false, false>(a, a.n_heads / a.kv.n_kv_heads, un)) return;
    stream_unit<D, KV8, NT, false>(a, un, lds);
}

// Joins the pieces of split tiles: RPW rows of a tile per workgroup, a thread per four dims of a row.
// Pieces' statistics and outputs load eight at a time.
template <int D, int RT>
__global__ void __launch_bounds__(256) attn_chunk_join_kernel(AttnChunkArgs a) {
    constexpr int RPW = 1024 / D, NS = RT / RPW;         // rows per workgroup; workgroups per tile
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<RT, true, false>(a, G, un)) return;
    const int rows = min(RT, un.sq.n * G - un.rt * RT);
    const int c = blockIdx.y * RPW + threadIdx.x / (D / 4), d0 = threadIdx.x % (D / 4) * 4;
    static_assert(NS * RPW == RT, "rows of a tile divide evenly");
    if (c >= rows) return;
    const int tiles = (un.sq.n * G + RT - 1) / RT;
    const float* src = a.ws + ((int64_t)un.part * RT + c) * wst(D);
    const int64_t step = (int64_t)tiles * RT * wst(D);
    float m = M0, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < un.pieces; i0 += 8) {
        float mi[8], li[8];
        f32x4 oi[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool on = i0 + j < un.pieces;
            const float* p = src + (i0 + j) * step;
            mi[j] = on ? p[D] : M0;
            li[j] = on ? p[D + 1] : 0.f;
            oi[j] = on ? *(const f32x4*)(p + d0) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
        float mn = m;
#pragma unroll
        for (int j = 0; j < 8; ++j) mn = fmaxf(mn, mi[j]);
        const float f = __builtin_amdgcn_exp2f(m - mn);
        l *= f;
        o *= f;
        m = mn;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float e = __builtin_amdgcn_exp2f(mi[j] - m);
            l += li[j] * e;
            o += oi[j] * e;
        }
    }
    const int rho = un.rt * RT + c;
    store4(a.out + ((int64_t)(un.sq.row0 + rho / G) * a.n_heads + un.kvh * G + rho % G) * D + d0, o * (1.f / l), a.out_fmt);
}

// Rows that a sequence can bring to a kv head decide the kernel: up to 64 go to the streaming kernel
// (tiles of 16, 32 or 64 rows), more to the tiles of 256.
int tile_rows(const fp_chunk& c, int G) {
    const int64_t R = (int64_t)std::min(c.max_new, c.n_rows) * G;
    return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : TILE_ROWS;
}

// log2 of the workgroups that run at a time (those of few rows: a half more), and the least number of blocks
// worth a piece
int piece_target(int RT, int D) { return RT == TILE_ROWS || (RT == 64 && D == 128) ? 8 : 9; }
int piece_min(int RT) { return RT == TILE_ROWS ? 8 : 16; }
// the most pieces that a call aims for (plan_q)
int64_t piece_aim(int RT, int D) { return (int64_t)1 << (piece_target(RT, D) + (RT < 64 ? 1 : 0)); }

}  // namespace

// Split tiles have more than Q blocks, so their pieces number at most twice total / Q, twice the aim.
size_t attn_chunk_ws_bytes(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    const int RT = tile_rows(c, n_heads / kv.n_kv_heads);
    return (size_t)(2 * piece_aim(RT, kv.head_dim)) * RT * wst(kv.head_dim) * sizeof(float);
}

template <int D, bool KV8, int RT>
static hipError_t launch_rt(AttnChunkArgs a, hipStream_t st) {
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    const int64_t tiles = std::min<int64_t>((int64_t)a.chunk.n_rows * G, (int64_t)a.chunk.n_rows * G / RT + a.chunk.n_seqs) * nkv;
    a.target = piece_target(RT, D);
    a.min_blocks = piece_min(RT);
    a.over = 10;
    a.join = 8;
    const int64_t pieces = piece_aim(RT, D), n = std::max(tiles + pieces, 2 * pieces) + 16;
    if (n > INT_MAX) return hipErrorInvalidValue;
    // tiles that can be split: each has more than Q of the blocks
    const unsigned split = (a.chunk.max_len + VT_BLK - 1) / VT_BLK <= a.min_blocks ? 0u : (unsigned)std::min<int64_t>(tiles, pieces);
    if constexpr (RT == TILE_ROWS) {
        return launch_attn_tile(a, (unsigned)n, split, st);
    } else {
        FP_LAUNCH((attn_chunk_kernel<D, KV8, RT / 16>), dim3((unsigned)n), dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || split == 0) return e;
        FP_LAUNCH((attn_chunk_join_kernel<D, RT>), dim3(split, RT * D / 1024), dim3(256), 0, st, a);
        return hipGetLastError();
    }
}

template <int D, bool KV8>
static hipError_t launch_d(const AttnChunkArgs& a, hipStream_t st) {
    switch (tile_rows(a.chunk, a.n_heads / a.kv.n_kv_heads)) {
        case 16: return launch_rt<D, KV8, 16>(a, st);
        case 32: return launch_rt<D, KV8, 32>(a, st);
        case 64: return launch_rt<D, KV8, 64>(a, st);
        default: return launch_rt<D, KV8, TILE_ROWS>(a, st);
    }
}

hipError_t launch_attn_chunk(const AttnChunkArgs& a, hipStream_t st) {
    const bool i8 = a.kv.format == FP_KV_INT8;
    if (a.kv.head_dim == 128) return i8 ? launch_d<128, true>(a, st) : launch_d<128, false>(a, st);
    if (a.kv.head_dim == 64) return i8 ? launch_d<64, true>(a, st) : launch_d<64, false>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace fpk
