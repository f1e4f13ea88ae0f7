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
// to the second product (vt_slot order).  int8: keys stay codes in bf16 (exact), a key's scale multiplies its
// scores and a value's its probabilities, which go to fp16 (11 bits; with the scale in them bf16's 8 would add to
// the codes' own error).  Online softmax per row in fp32, base 2.  (attn_stream.h: a unit's work.)
//
// Many rows to a kv head take tiles of 256 (attn_tile.hip; tile_rows below has the rule): there the matrix cores
// bound, here the reads of the cache.
//
// Work is split over the keys: from the lengths in device memory every workgroup works out the same plan, or for more than
// 256 sequences a kernel before it (attn_plan.h).  A piece is (sequence, kv head, row tile, a run of 32-key blocks); its four waves take every
// fourth block and merge in LDS.  A tile of one piece is written out at once; the pieces of the others
// go to the workspace as unnormalised (o, m, l) and a second kernel joins them in order:
//     m = max m_i,  l = sum l_i 2^(m_i - m),  o = sum o_i 2^(m_i - m) / l.
// The plan depends on the inputs alone, so results repeat bit for bit.
//
// Next tokens of 32 sequences of 4096, 8 kv heads of 128 (268 MB of cache): bf16, 8 rows 50 us (5.3 TB/s, the
// rate of a large copy), 24 rows 53, 48 rows 70; int8 31, 37, 68.  One sequence of 331 positions, 32 kv heads: 9.7 us, of
// which 1.4 are the plan, 1.3 the first loads, 4 three blocks a wave and 1.8 the merge (a chain of memory latencies
// and of code fetched for the first time: a second copy of the block's code cost 1 us).
#include "attn_stream.h"

namespace fpk {

namespace {

template <int D, bool KV8, int NT, bool TREE>
__global__ void __launch_bounds__(256, NT == 1 ? 3 : NT == 4 && D == 128 ? 1 : 2) attn_chunk_kernel(AttnChunkArgs a) {
    __shared__ StreamLds<D, NT, TREE> lds;
    Unit un;
    if (!find_unit<16 * NT, false, false>(a, a.n_heads / a.kv.n_kv_heads, un)) return;
    stream_unit<D, KV8, NT, false, TREE>(a, un, lds);
}

// The plan of more than 256 sequences (attn_plan.h), by one workgroup: PER sequences a thread, their sums and running
// counts over the waves.  Next tokens of 1024 sequences of up to 200, 8 heads of 128, bf16: 138 us with it, of which it takes
// 5; 306 with every workgroup planning for itself.  4096 sequences: 496, 2988.
constexpr int PLAN_T = 1024, PER = 4096 / PLAN_T;
template <int RT>
__global__ void __launch_bounds__(PLAN_T) attn_plan_kernel(AttnChunkArgs a) {
    constexpr int W = PLAN_T / 64;
    __shared__ int64_t st[W];
    __shared__ int sn[W], sc[4][W];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Seq sq[PER];
    int64_t total = 0;
    int tiles = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        sq[i] = b < a.chunk.n_seqs ? load_seq(a.chunk, b) : Seq{0, 0, 0, 0};
        const Plan p = plan_seq<RT>(sq[i], G, 1);
        total += (int64_t)p.tiles * p.blocks;
        tiles = std::min(tiles + long_tiles<RT>(sq[i], G, p), 1 << 20);
    }
    total = std::min(total, TOTAL_MAX);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        total += __shfl_xor(total, o, 64);
        tiles = std::min(tiles + __shfl_xor(tiles, o, 64), 1 << 24);
    }
    if (lane == 0) {
        st[w] = total;
        sn[w] = tiles;
    }
    __syncthreads();
    total = 0;
    tiles = 0;
    for (int j = 0; j < W; ++j) {
        total += st[j];
        tiles += sn[j];
    }
    const int Q = plan_all<RT>(a, total, tiles);
    int mine[4] = {0, 0, 0, 0}, base[4];
    PlanRow row[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        row[i] = plan_row<RT, RT == TILE_ROWS>(sq[i], G, nkv, Q);
        mine[0] += row[i].units;
        mine[1] += row[i].few;
        mine[2] += row[i].split;
        mine[3] += row[i].part;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        base[k] = wave_scan(mine[k]);
        if (lane == 63) sc[k][w] = base[k];
        base[k] -= mine[k];
    }
    __syncthreads();
    int all[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        all[k] = 0;
        for (int j = 0; j < W; ++j) {
            base[k] += j < w ? sc[k][j] : 0;
            all[k] += sc[k][j];
        }
    }
    PlanRow* rows = (PlanRow*)(a.plan + PLAN_HEAD);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        if (b < a.chunk.n_seqs) rows[b] = PlanRow{base[0], base[1], base[2], base[3]};
        base[0] += row[i].units;
        base[1] += row[i].few;
        base[2] += row[i].split;
        base[3] += row[i].part;
    }
    if (tid == 0) {
        a.plan[PLAN_Q] = Q;
        a.plan[PLAN_UNITS] = all[0];
        a.plan[PLAN_FEW] = all[1];
        a.plan[PLAN_SPLIT] = all[2];
    }
}

// Joins the pieces of split tiles: RPW rows of a tile at a time, a thread per four dims of a row.  Pieces' statistics and
// outputs load GRP at a time.  Wide tiles, whose pieces are two or three, four times per workgroup (each has to find its tile first)
// and without a branch around a load (48 sequences of up to 3000, 14 nodes, 64 heads on 8, int8: with its attention 98.5 us, so 94.5;
// 32 of up to 8192, 16 nodes 141, 138).
constexpr int join_reps(int tile) { return tile & WIDE ? 4 : 1; }
template <int D, int TILE>
__global__ void __launch_bounds__(256) attn_chunk_join_kernel(AttnChunkArgs a) {
    constexpr bool ALL = (TILE & WIDE) != 0;
    constexpr int RT = tile_size(TILE), RPW = 1024 / D, REP = join_reps(TILE), GRP = ALL ? 4 : 8;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<TILE, true, false>(a, G, un)) return;
    const int rows = min(RT, un.sq.n * G - un.rt * RT);
    const int c0 = blockIdx.y * (RPW * REP) + threadIdx.x / (D / 4), d0 = threadIdx.x % (D / 4) * 4;
    static_assert(RT % (RPW * REP) == 0, "rows of a tile divide evenly");
    const int tiles = (un.sq.n * G + RT - 1) / RT;
    const int64_t step = (int64_t)tiles * RT * wst(D);
#pragma unroll
    for (int k = 0; k < REP; ++k) {
        const int c = c0 + k * RPW;
        if (c >= rows) return;
        const float* src = a.ws + ((int64_t)un.part * RT + c) * wst(D);
        float m = M0, l = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i0 = 0; i0 < un.pieces; i0 += GRP) {
            float mi[GRP], li[GRP];
            f32x4 oi[GRP];
#pragma unroll
            for (int j = 0; j < GRP; ++j) {
                const bool on = i0 + j < un.pieces;
                const float* p = src + (ALL ? min(i0 + j, un.pieces - 1) : i0 + j) * step;
                const f32x2 ml = ALL || on ? *(const f32x2*)(p + D) : f32x2{M0, 0.f};
                const f32x4 x = ALL || on ? *(const f32x4*)(p + d0) : f32x4{0.f, 0.f, 0.f, 0.f};
                mi[j] = on ? ml.x : M0;
                li[j] = on ? ml.y : 0.f;
                oi[j] = on ? x : f32x4{0.f, 0.f, 0.f, 0.f};
            }
            float mn = m;
#pragma unroll
            for (int j = 0; j < GRP; ++j) mn = fmaxf(mn, mi[j]);
            const float f = __builtin_amdgcn_exp2f(m - mn);
            l *= f;
            o *= f;
            m = mn;
#pragma unroll
            for (int j = 0; j < GRP; ++j) {
                const float e = __builtin_amdgcn_exp2f(mi[j] - m);
                l += li[j] * e;
                o += oi[j] * e;
            }
        }
        const int rho = un.rt * RT + c;
        store4(a.out + ((int64_t)(un.sq.row0 + rho / G) * a.n_heads + un.kvh * G + rho % G) * D + d0, o * (1.f / l), a.out_fmt);
    }
}

// Rows of a tile, by what a sequence can bring to a kv head and by the call's size: 64-row tiles times the blocks that
// they can see.  us at (new tokens after context), 8 heads a kv head, unless said otherwise.
//   More than 64 rows: tiles of 256, where the matrix cores bound, once they fill the GPU and their longer start pays.
// Streamed and in tiles of 256:
//     d 128, bf16   up to 2^13: 512 after 0 21, 34; 512 after 512 32, 35    above: 1024 after 0 61, 47; 1024 after 31744 832, 523
//     d 64, bf16    up to 2^15: 1024 after 0 32, 35; 128 after 16000 40, 46    above: 2048 after 0 71, 60; 1024 after 31744 391, 360
//     d 64, int8    always: 512 after 0 14, 33; 2048 after 0 77, 83; 8 sequences of 2048 after 2000 505, 551; 1024 after
//                   31744 554, 523 (the tiles' unpacking costs as much as their products)
//   Streamed, more than 32 rows: tiles of 64 read the cache once for them all, tiles of 32 start and end sooner and
// two or three waves a SIMD hide each other's waits.  In tiles of 64 and of 32:
//     small calls, or up to 8 blocks: 256 after 0 d 128 16, 11; d 64 11, 8; 5 after 2000 d 128 bf16 23, 16
//     int8 of 128 dims, up to 64 rows: 5 of 64 sequences after up to 2000 84, 75; 4 after 300, 16 heads a kv head 16, 10
//     others: 5 of 16 sequences after up to 4000, d 128 bf16 36, 52; 512 after 512 32, 47; 6 of 32 after up to 4096, d 64 int8
//     37, 42
int tile_rows(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    const int64_t G = n_heads / kv.n_kv_heads, R = std::min(c.max_new, c.n_rows) * G;
    if (R <= 32) return R <= 16 ? 16 : 32;
    const int blocks = (c.max_len - 1) / VT_BLK + 1;
    const double work = (double)((c.n_rows * G + 63) / 64) * kv.n_kv_heads * blocks;
    const bool i8 = kv.format == FP_KV_INT8;
    if (R > 64 && !(kv.head_dim == 64 && i8) && work > (kv.head_dim == 128 ? 8192.0 : 32768.0)) return TILE_ROWS;
    if (i8 && kv.head_dim == 128 && R <= 64) return 32;
    return blocks <= 8 || work <= (i8 ? 4096.0 : 2048.0) ? 32 : 64;
}

// The same for trees: as chunks, but for more than 64 rows of 128 dims.  us, 64 heads on 8 (G: heads of a group):
//   65 to 128 rows, a tree's most common number, take tiles of 128 (attn_wide.hip) in large calls: 16 nodes of 32 sequences of up to 8192
// bf16 140, in tiles of 256 225, of 64 216; int8 143, 279, of 32 202.  int8 with less than half a tile a sequence only above 96 blocks
// (up to 12 nodes of 64 sequences of 2000, in tiles of 128 95, of 32 82; of 48 of up to 3000 94, 94; of 24 of up to 8192 96, 106).
//   Whole tiles of 128 (nothing to join, no room for pieces needed) where they fill half of the CUs: 16 nodes of 32 sequences of 250, int8
// 22, in tiles of 64 37, of 32 30; of 16 sequences 20, 17, 17.  With more than 128 rows, above 8 blocks: 32 nodes of 16 sequences of 500, int8
// 26, in tiles of 256 48; and, more of them than run at once, where sequences have fewer rows than the most: up to 32 nodes of 64 sequences of 900 92,
// in tiles of 256 115; 32 nodes of each 109, 119; bf16 104, 99; 20 of 64 of 300 int8 70, 58.
//   The rest: tiles of 32 instead of 64, which hold a CU each: 23 nodes of 17 sequences of up to 1777, G 4, int8 45, of 32 29;
// bf16 42, 36; up to 32 of 8 of 900, int8 41, 28.  Not bf16 calls whose tiles of 64 run at once: 4 sequences of 4000, 16 nodes, 28, 32.
// (Long contexts with 256 rows and more, in pairs of tiles of 128 or tiles of 256 made the same way: no faster than attn_tile.hip's, 8 sequences
// of up to 30001 with 512 rows to a kv head, bf16 69 and 61 against 61.  48 rows: int8 183, in tiles of 32 94; bf16 161, in tiles of 64 134.)
int tree_rows(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    const int RT = tile_rows(kv, c, n_heads), blocks = (c.max_len - 1) / VT_BLK + 1;
    const int64_t G = n_heads / kv.n_kv_heads, R = std::min(c.max_new, c.n_rows) * G, n_seqs = std::min(c.n_seqs, c.n_rows);
    if (kv.head_dim != 128 || R <= 64) return RT;
    const bool i8 = kv.format == FP_KV_INT8, half = c.n_rows * G >= 64 * n_seqs;
    const bool whole = blocks <= WHOLE<WIDE | 128> && c.n_rows * G * kv.n_kv_heads > 128 * 128;
    if (R > 128) {
        const bool ragged = 4 * (int64_t)c.n_rows < 3 * n_seqs * c.max_new, at_once = (R + 127) / 128 * n_seqs * kv.n_kv_heads <= 256;
        if (whole && blocks > 8 && (RT != TILE_ROWS || ragged || at_once)) return WIDE | 128;
        if (RT == TILE_ROWS) return RT;
    } else {
        if (half && (whole || RT == TILE_ROWS)) return WIDE | 128;
        if (RT == TILE_ROWS) return i8 && blocks <= 96 ? 32 : WIDE | 128;
    }
    return i8 || (R + 63) / 64 * n_seqs * kv.n_kv_heads > 256 ? 32 : RT;
}

// log2 of the workgroups that run at a time (those of few rows: a half more), and the least number of blocks
// worth a piece
int piece_target(int RT, int D) { return RT == TILE_ROWS || (RT == 64 && D == 128) ? 8 : 9; }
int piece_min(int RT) { return RT == TILE_ROWS ? 8 : 16; }
// the most pieces that a call aims for (plan_one, plan_all)
int64_t piece_aim(int RT, int D) { return (int64_t)1 << (piece_target(RT, D) + (RT < 64 ? 1 : 0)); }

}  // namespace

// Split tiles have more than Q blocks, so their pieces number at most twice total / Q, twice the aim.  Enough for
// calls of smaller bounds too, whose tiles may be smaller, and for those of trees in wide tiles.
static_assert(WIDE_PIECES * 128 <= 2 * TILE_ROWS * TILE_ROWS, "WIDE_PIECES fit where tiles of 256 rows do");
size_t attn_chunk_ws_bytes(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    int64_t rows = 0;
    for (const int RT : {16, 32, 64, TILE_ROWS})
        if (RT <= tile_rows(kv, c, n_heads)) rows = std::max(rows, 2 * piece_aim(RT, kv.head_dim) * RT);
    return (size_t)rows * wst(kv.head_dim) * sizeof(float) + (size_t)plan_ints(c.n_seqs) * sizeof(int);
}

template <int D, bool KV8, int RT>
static hipError_t launch_rt(AttnChunkArgs a, hipStream_t st) {
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    // rows that sequences own, which may be few of a padded batch's
    const int64_t R = std::min<int64_t>(a.chunk.n_rows, (int64_t)a.chunk.n_seqs * a.chunk.max_new) * G;
    const int64_t tiles = std::min(R, R / RT + a.chunk.n_seqs) * nkv;
    a.target = piece_target(RT, D);
    a.min_blocks = piece_min(RT);
    a.over = 10;
    a.join = 8;
    a.plan = (int*)(a.ws + 2 * piece_aim(RT, D) * RT * wst(D));
    const int64_t pieces = piece_aim(RT, D), n = std::max(tiles + pieces, 2 * pieces) + 16 * XCD_RUN;
    if (n > MAX_GRID) return hipErrorInvalidValue;
    // tiles that can be split: each has more than Q of the blocks
    const unsigned split = (a.chunk.max_len - 1) / VT_BLK < WHOLE<RT> ? 0u : (unsigned)std::min<int64_t>(tiles, pieces);
    if (a.chunk.n_seqs > PLAN_LANES) {
        FP_LAUNCH(attn_plan_kernel<RT>, dim3(1), dim3(PLAN_T), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if constexpr (RT == TILE_ROWS) {
        return launch_attn_tile(a, (unsigned)n, split, st);
    } else {
        if (a.parent != nullptr) FP_LAUNCH((attn_chunk_kernel<D, KV8, RT / 16, true>), dim3((unsigned)n), dim3(256), 0, st, a);
        else FP_LAUNCH((attn_chunk_kernel<D, KV8, RT / 16, false>), dim3((unsigned)n), dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || split == 0) return e;
        FP_LAUNCH((attn_chunk_join_kernel<D, RT>), dim3(split, RT * D / 1024), dim3(256), 0, st, a);
        return hipGetLastError();
    }
}

// Trees in wide tiles.
static hipError_t launch_wide(AttnChunkArgs a, hipStream_t st) {
    constexpr int RT = WIDE | 128, D = 128;
    const int64_t nkv = a.kv.n_kv_heads, R = std::min<int64_t>(a.chunk.n_rows, (int64_t)a.chunk.n_seqs * a.chunk.max_new) * (a.n_heads / nkv);
    const int64_t tiles = std::min(R, R / 128 + a.chunk.n_seqs) * nkv, n = tiles + WIDE_PIECES + 8 * XCD_RUN;
    a.min_blocks = 32;
    if (n > MAX_GRID) return hipErrorInvalidValue;
    const unsigned split = (a.chunk.max_len - 1) / VT_BLK < WHOLE<RT> ? 0u : (unsigned)std::min<int64_t>(tiles, WIDE_PIECES);
    a.plan = (int*)(a.ws + (split > 0 ? (int64_t)WIDE_PIECES * 128 * wst(D) : 0));      // (whole tiles leave no pieces)
    hipError_t e;
    if (a.chunk.n_seqs > PLAN_LANES) {
        FP_LAUNCH(attn_plan_kernel<RT>, dim3(1), dim3(PLAN_T), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if ((e = launch_attn_wide(a, (unsigned)n, st)) != hipSuccess || split == 0) return e;
    FP_LAUNCH((attn_chunk_join_kernel<D, RT>), dim3(split, 128 * D / 1024 / join_reps(RT)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int D, bool KV8>
static hipError_t launch_d(const AttnChunkArgs& a, hipStream_t st) {
    const int RT = a.parent != nullptr ? tree_rows(a.kv, a.chunk, a.n_heads) : tile_rows(a.kv, a.chunk, a.n_heads);
    if (RT & WIDE) return launch_wide(a, st);
    switch (RT) {
        case 16: return launch_rt<D, KV8, 16>(a, st);
        case 32: return launch_rt<D, KV8, 32>(a, st);
        case 64: return launch_rt<D, KV8, 64>(a, st);
    }
    if constexpr (D == 64 && KV8) return hipErrorInvalidValue;
    else return launch_rt<D, KV8, TILE_ROWS>(a, st);
}

hipError_t launch_attn_chunk(const AttnChunkArgs& a, hipStream_t st) {
    const bool i8 = a.kv.format == FP_KV_INT8;
    if (a.kv.head_dim == 128) return i8 ? launch_d<128, true>(a, st) : launch_d<128, false>(a, st);
    if (a.kv.head_dim == 64) return i8 ? launch_d<64, true>(a, st) : launch_d<64, false>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace fpk
