// Work plan of the chunk attention, made by every workgroup from the lengths in device memory, and what
// its kernels share.
#pragma once
#include <algorithm>

#include "paged.h"

namespace fpk {

struct Plan {
    int tiles, blocks, pieces;             // row tiles, 32-key blocks, pieces per tile
};
__device__ __forceinline__ Plan plan_seq(const Seq& s, int G, int RT, int Q) {
    Plan p;
    p.tiles = (s.n * G + RT - 1) / RT;
    p.blocks = s.n > 0 ? (s.len + VT_BLK - 1) / VT_BLK : 0;
    p.pieces = (p.blocks + Q - 1) / Q;
    return p;
}

// The chunk's sequences across a wave's lanes, 64 at a time: f(b, sequence) for lane's b of each
// round.  The first 64 are loaded once and kept.
struct Lanes {
    const fp_chunk& c;
    Seq s0;
    __device__ __forceinline__ explicit Lanes(const fp_chunk& ch) : c(ch) { s0 = at(0); }
    __device__ __forceinline__ Seq at(int b0) const {
        const int b = b0 + (int)(threadIdx.x & 63);
        return b < c.n_seqs ? load_seq(c, b) : Seq{0, 0, 0, 0};
    }
    __device__ __forceinline__ Seq get(int b0) const { return b0 == 0 ? s0 : at(b0); }
};
// Blocks per piece, Q: about the total over 2^a.target, and at least a.min_blocks.  Where few workgroups run at
// a time (2^a.slots > 1) and there is one sequence, whose pieces are all alike, a last round of a few pieces
// would cost as much as a full one: its tiles are cut so that the pieces just fill one round, or two, or not
// at all, whichever costs least: rounds times (blocks of a piece + a.over, a piece's fixed part), and a.join
// for joining, all in blocks.  Several sequences' pieces differ in size and fill each other's gaps: there the aim
// is lowered by half a piece a tile, which rounding up adds, so that one round holds them.
// Totals are summed in halves of 24 bits, so that 64 lanes' sums fit.
__device__ __forceinline__ int plan_q(const AttnChunkArgs& a, const Lanes& L, int G, int RT) {
    if (a.slots > 0 && a.chunk.n_seqs == 1) {
        const Seq s{__builtin_amdgcn_readfirstlane(L.s0.row0), __builtin_amdgcn_readfirstlane(L.s0.n),
                    __builtin_amdgcn_readfirstlane(L.s0.ctx), __builtin_amdgcn_readfirstlane(L.s0.len)};
        const Plan p = plan_seq(s, G, RT, 1);
        const int tiles = std::max(1, p.tiles * a.kv.n_kv_heads);        // above 2^31 the launch is refused
        int best = std::max(1, p.blocks), cost = ((tiles - 1 >> a.slots) + 1) * (p.blocks + a.over);
        for (int k = 0; k < 2; ++k) {
            const int cut = std::min((1 << (a.slots + k)) / tiles, p.blocks / a.min_blocks);
            if (cut < 2) continue;
            const int Q = (p.blocks + cut - 1) / cut;
            const int c = ((tiles * cut - 1 >> a.slots) + 1) * (Q + a.over) + a.join;
            if (c < cost) {
                cost = c;
                best = Q;
            }
        }
        return best;
    }
    int64_t total = 0;
    int tiles = 0;
    for (int b0 = 0; b0 < a.chunk.n_seqs; b0 += 64) {
        const Plan p = plan_seq(L.get(b0), G, RT, 1);
        const int64_t t = (int64_t)p.tiles * p.blocks;
        if (a.slots > 0) tiles += std::min(wave_total(p.tiles), 1 << 20);
        total += wave_total((int)(t & 0xFFFFFF)) + ((int64_t)wave_total((int)(t >> 24)) << 24);
    }
    total *= a.kv.n_kv_heads;
    if (a.slots > 0) {
        const float aim = fmaxf((float)(1 << a.target) - 0.5f * (float)tiles * (float)a.kv.n_kv_heads, 0.5f * (float)(1 << a.target));
        return std::max(a.min_blocks, (int)fminf((float)total / aim, 1.6e7f) + 1);
    }
    total = (total + ((int64_t)1 << a.target) - 1) >> a.target;
    return std::max(a.min_blocks, (int)std::min<int64_t>(total, 1 << 24));
}

// What a workgroup works on: row tile rt of kv head kvh of sequence b, blocks beg .. end - 1 (one of
// `pieces` of the tile's), and the place of its partial result among all split tiles' pieces.
struct Unit {
    Seq sq;
    int b, kvh, rt, beg, end, pieces, part;
};
// Unit u, or false if there are not that many.  SPLIT: u counts the split tiles instead, and the unit
// is the tile's first piece.  XCD: consecutive units (the row tiles that read the same keys) go to one
// XCD's workgroups (workgroup i runs on XCD i % 8).
template <bool SPLIT, bool XCD>
__device__ __forceinline__ bool find_unit(const AttnChunkArgs& a, int G, int RT, Unit& un) {
    const int nkv = a.kv.n_kv_heads, lane = threadIdx.x & 63;
    const Lanes L(a.chunk);
    const int Q = plan_q(a, L, G, RT);
    auto units = [&](const Plan& p) { return SPLIT ? (p.pieces > 1 ? p.tiles * nkv : 0) : p.tiles * p.pieces * nkv; };
    int u = blockIdx.x;
    if constexpr (XCD) {
        int all = 0;
        for (int b0 = 0; b0 < a.chunk.n_seqs; b0 += 64) all += wave_total(units(plan_seq(L.get(b0), G, RT, Q)));
        const int per = (all + 7) / 8;
        if (u >> 3 >= per) return false;
        u = (u & 7) * per + (u >> 3);
    }
    int part = 0;
    un.b = -1;
    for (int b0 = 0; b0 < a.chunk.n_seqs; b0 += 64) {
        const Seq lane_seq = L.get(b0);
        const Plan p = plan_seq(lane_seq, G, RT, Q);
        const int c = units(p), sp = p.pieces > 1 ? p.tiles * p.pieces * nkv : 0;
        const int s = wave_scan(c);
        const uint64_t past = __ballot(s > u);
        if (past) {
            const int l = __builtin_ctzll(past);
            u -= __builtin_amdgcn_readlane(s - c, l);
            part += wave_total(lane < l ? sp : 0);
            un.b = b0 + l;
            un.sq = Seq{__builtin_amdgcn_readlane(lane_seq.row0, l), __builtin_amdgcn_readlane(lane_seq.n, l),
                        __builtin_amdgcn_readlane(lane_seq.ctx, l), __builtin_amdgcn_readlane(lane_seq.len, l)};
            break;
        }
        u -= __builtin_amdgcn_readlane(s, 63);
        part += wave_total(sp);
    }
    if (un.b < 0) return false;
    const Plan pl = plan_seq(un.sq, G, RT, Q);
    if (u < 0 || u >= units(pl)) return false;         // overlapping rows: sums past int32
    un.pieces = pl.pieces;
    un.rt = u % pl.tiles;
    const int v = u / pl.tiles, sp = SPLIT ? 0 : v % pl.pieces;
    un.kvh = SPLIT ? v : v / pl.pieces;
    un.part = part + (SPLIT ? un.kvh * pl.pieces * pl.tiles + un.rt : u);
    const int per = (pl.blocks + pl.pieces - 1) / pl.pieces;
    // no further than the tile's last row sees
    const int last = min((un.rt + 1) * RT, un.sq.n * G) - 1;
    un.beg = sp * per;
    un.end = min(min(un.beg + per, pl.blocks), (un.sq.ctx + last / G) / VT_BLK + 1);
    return true;
}

// Slots of a value block are keys 16 (x / 2) + 4 g + 2 (x % 2), + 1 in word x of the eight of chunk g:
// the bits of those below key n.
__device__ __forceinline__ uint32_t slots_below(int g, int x, int n) {
    const int key = 16 * (x >> 1) + 4 * g + 2 * (x & 1);
    return (key < n ? 0x0000FFFFu : 0u) | (key + 1 < n ? 0xFFFF0000u : 0u);
}
// The high bits of the halves of w whose exponent bits E are all ones.
template <uint32_t E>
__device__ __forceinline__ uint32_t nonfinite(uint32_t w) {
    constexpr uint32_t M = E * 0x10001u, A = (0x8000u - E) * 0x10001u;
    return ((w & M) + A) & 0x80008000u;
}
constexpr uint32_t BF16_EXP = 0x7F80u, F16_EXP = 0x7C00u;
// w with those halves zero
template <uint32_t E>
__device__ __forceinline__ uint32_t finite_halves(uint32_t w) {
    return w & ~((nonfinite<E>(w) >> 15) * 0xFFFFu);
}

// Infinite and NaN values that some rows of a tile do not see would make NaN of their zero probabilities.
// The kernels take them out of the products; this is what they are to a row that sees them: the sum of those of
// dim d at positions first .. last, 0 if there are none (rare, and not quick).
template <int D, bool KV8>
__device__ __forceinline__ float stray_sum(const AttnChunkArgs& a, int b, int kvh, int d, int first, int last) {
    float sum = 0.f;
    for (int p = first; p <= last; ++p) {
        const int pb = pool_block(a.kv, a.chunk, b, kvh, p / VT_BLK), t = p % VT_BLK;
        if (pb < 0) continue;
        const int64_t at = ((int64_t)pb * D + d) * VT_BLK + vt_slot(t);
        float v;
        if constexpr (KV8) v = (float)((const int8_t*)a.kv.v)[at] * h2f(((const uint16_t*)a.kv.v_scales)[(int64_t)pb * VT_BLK + t]);
        else v = __uint_as_float((uint32_t)((const uint16_t*)a.kv.v)[at] << 16);
        if (!(fabsf(v) < INFINITY)) sum += v;
    }
    return sum;
}

constexpr int wst(int D) { return D + 4; }     // floats per row of a piece: o, then m, l

__device__ __forceinline__ void store4(uint16_t* p, f32x4 v, int fmt) {
    uint16_t x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = act_store((float)(__bf16)v[e], fmt);
    *(u32x2*)p = u32x2{(uint32_t)x[0] | ((uint32_t)x[1] << 16), (uint32_t)x[2] | ((uint32_t)x[3] << 16)};
}

constexpr int TILE_ROWS = 256;             // rows per tile of attn_tile.hip
constexpr float M0 = -3e38f;               // softmax reference before any score

}  // namespace fpk
