// Work plan of the chunk attention, made on the device from the lengths there, and what its kernels share.
#pragma once
#include <algorithm>

#include "paged.h"

namespace fpk {

typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int TILE_ROWS = 256;             // rows per tile of attn_tile.hip
constexpr float M0 = -3e38f;               // softmax reference before any score

// Sequences with at most 16 rows to a kv head in a call of 256-row tiles (next tokens beside a prompt's chunk)
// are streamed like those of a call without larger ones.
__device__ __forceinline__ bool few_rows(const Seq& s, int G) { return s.n * G <= 16; }

// Scores are scaled as |scale| (q with its signs turned for a negative scale).  A scale of zero, or too small to
// matter, would make NaN of a masked score's -infinity: the queries are zero then, and the scale one.
struct QScale {
    float sl2;                             // |scale| log2 e
    uint32_t sign, keep;                   // of two bf16 or fp16 queries: (q ^ sign) & keep
};
__device__ __forceinline__ QScale q_scale(float scale) {
    const bool none = fabsf(scale) < 1.2e-38f;
    return QScale{none ? 1.f : fabsf(scale) * 1.4426950408889634f, scale < 0.f ? 0x80008000u : 0u, none ? 0u : 0xFFFFFFFFu};
}

struct Plan {
    int tiles, blocks, pieces;             // row tiles, 32-key blocks, pieces per tile
};
// A tile of so few blocks is not split: joining costs as much as they do.  (Streamed, 600 positions, 8 kv heads of 128, bf16:
// 64 sequences 22 us whole, 26 in two pieces; one sequence of 1000 17, 15.  Tiles of 256, 4 prompts of 512, 32 heads of 128, bf16
// 37 whole, 47 in two.)
template <int RT>
constexpr int WHOLE = RT == TILE_ROWS ? 16 : RT == 64 ? 20 : 24;
template <int RT>
__device__ __forceinline__ Plan plan_seq(const Seq& s, int G, int Q) {
    Plan p;
    p.tiles = (s.n * G + RT - 1) / RT;
    p.blocks = s.n > 0 ? (s.len - 1) / VT_BLK + 1 : 0;
    p.pieces = p.blocks <= WHOLE<RT> ? std::min(p.blocks, 1) : (p.blocks + Q - 1) / Q;
    return p;
}

// Blocks per piece, Q: the total over the pieces to aim for, and at least a.min_blocks.  2^a.target workgroups or so
// run at a time.
// One sequence's pieces are all alike.  Of 64 rows and more, a last round of a few pieces would cost as much
// as a full one: its tiles are cut so that the pieces just fill one round, or two, or not at all, whichever
// costs least: rounds times (blocks of a piece + a.over, a piece's fixed part), and a.join for joining, all in
// blocks.  Fewer rows stream at the memory's rate however the rounds fall.
// Several sequences' pieces differ in size and fill each other's gaps: there the aim is lowered by half a piece
// a tile, which rounding up adds, so that one round holds them.  Tiles of few rows that fill the round by themselves are
// cut for two.  (Next tokens of 32 sequences of 16384: int8, 8 kv heads 106 us; aiming for 512 or 1024 whatever the tiles 118,
// 111.  bf16, 32 kv heads 717; lowered there too 791.)
template <int RT>
__device__ __forceinline__ int plan_one(const AttnChunkArgs& a, const Seq& s, int G) {
    const Plan p = plan_seq<RT>(s, G, 1);
    const int tiles = std::max(1, p.tiles * a.kv.n_kv_heads);        // above MAX_GRID the launch is refused
    int best = std::max(1, p.blocks), cost = ((tiles - 1 >> a.target) + 1) * (p.blocks + a.over);
    for (int k = 0; k < 2; ++k) {
        const int cut = std::min((1 << (a.target + k)) / tiles, p.blocks / a.min_blocks);
        if (cut < 2) continue;
        const int Q = (p.blocks + cut - 1) / cut;
        const int c = ((tiles * cut - 1 >> a.target) + 1) * (Q + a.over) + a.join;
        if (c < cost) {
            cost = c;
            best = Q;
        }
    }
    return best;
}
// A count of TOTAL_MAX leaves every tile whole, as a larger one does: rows that overlap cannot overflow the sums.
constexpr int64_t TOTAL_MAX = (int64_t)1 << 40;
// total: tiles times blocks of all sequences; tiles: those not of few rows.  Both of one kv head.
template <int RT>
__device__ __forceinline__ int plan_all(const AttnChunkArgs& a, int64_t total, int tiles) {
    const float round = (float)(1 << a.target), nt = (float)tiles * (float)a.kv.n_kv_heads;
    float aim = fmaxf(round - 0.5f * nt, 0.5f * round);
    if (RT < 64 && a.chunk.n_seqs == 1) aim = round;
    if (RT < 64 && nt >= round) aim = 2.f * round;
    const float q = (float)total * (float)a.kv.n_kv_heads / aim;
    return std::max(a.min_blocks, (int)fminf(q, 2.5e8f) + 1);        // above any sequence's blocks
}
template <int RT>
__device__ __forceinline__ int long_tiles(const Seq& s, int G, const Plan& p) {
    return RT == TILE_ROWS && few_rows(s, G) ? 0 : p.tiles;
}

// Up to 256 sequences every workgroup plans for itself, up to four sequences a lane.  For more a kernel of its own does it
// first (attn_plan_kernel, 5 us), and leaves Q, the totals and per sequence the running counts in a.plan:
enum { PLAN_Q, PLAN_UNITS, PLAN_FEW, PLAN_SPLIT, PLAN_HEAD };        // totals: units, those of few rows, split tiles
struct PlanRow {
    int units, few, split, part;           // of the sequences before: units (of many rows, of few), split tiles, their pieces
};
constexpr int PER_LANE = 4, PLAN_LANES = 64 * PER_LANE;
constexpr int64_t plan_ints(int n_seqs) { return n_seqs > PLAN_LANES ? PLAN_HEAD + 4 * (int64_t)n_seqs : 0; }

// What a sequence adds to the running counts.
template <int RT, bool SORT>
__device__ __forceinline__ PlanRow plan_row(const Seq& s, int G, int nkv, int Q) {
    const Plan p = plan_seq<RT>(s, G, Q);
    const int u = p.tiles * p.pieces * nkv;
    const bool few = SORT && few_rows(s, G), split = p.pieces > 1;
    return PlanRow{few ? 0 : u, few ? u : 0, split ? p.tiles * nkv : 0, split ? u : 0};
}

// What a workgroup works on: row tile rt of kv head kvh of sequence b, blocks beg .. end - 1 (one of
// `pieces` of the tile's), and the place of its partial result among all split tiles' pieces.
struct Unit {
    Seq sq;
    int b, kvh, rt, beg, end, pieces, part;
};
// A workgroup's place among the units by a plan's totals: the unit, and whether it is one of few rows.  False past the last.
// SPLIT: the split tiles are counted instead.  SORT: XCD_RUN consecutive units (row tiles that read the same keys) go to one
// XCD's workgroups (workgroup i runs on XCD i % 8), and those of sequences with few rows, which are short, come last.
constexpr int XCD_RUN = 4;
template <bool SPLIT, bool SORT>
__device__ __forceinline__ bool place(int units, int few, int split, int& u, bool& last) {
    u = blockIdx.x;
    last = false;
    if constexpr (SORT) {
        constexpr int R = 8 * XCD_RUN;
        const int first = (units + R - 1) / R * R;
        last = u >= first;
        if (last) u -= first;
        u = u / R * R + u % 8 * XCD_RUN + u % R / 8;
    }
    return u >= 0 && u < (SPLIT ? split : last ? few : units);
}
template <bool SPLIT>
__device__ __forceinline__ int counted(const PlanRow& w, bool last) { return SPLIT ? w.split : last ? w.few : w.units; }

// Sequence, unit in it and pieces of the split tiles before it, for up to 64 PER sequences: lane l has PER l .. PER l + PER - 1.
template <int RT, bool SPLIT, bool SORT, int PER>
__device__ __forceinline__ bool find_by_lanes(const AttnChunkArgs& a, int G, Unit& un, int& Q, int& u, int& part) {
    constexpr bool CLASSES = RT == TILE_ROWS;            // as the plan counts them
    const int nkv = a.kv.n_kv_heads, lane = threadIdx.x & 63, n_seqs = a.chunk.n_seqs;
    Seq mine[PER];
    PlanRow row[PER], sum{0, 0, 0, 0};
    int64_t t = 0;                                       // summed in halves of 24 bits
    int tiles = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = PER * lane + i;
        mine[i] = b < n_seqs ? load_seq(a.chunk, b) : Seq{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const Plan p = plan_seq<RT>(mine[i], G, 1);
        t += (int64_t)p.tiles * p.blocks;
        tiles += long_tiles<RT>(mine[i], G, p);
    }
    t = std::min(t, TOTAL_MAX);
    if (PER == 1 && RT >= 64 && n_seqs == 1) Q = plan_one<RT>(a, lane_seq(mine[0], 0), G);
    else Q = plan_all<RT>(a, wave_total((int)(t & 0xFFFFFF)) + ((int64_t)wave_total((int)(t >> 24)) << 24),
                          std::min(wave_total(tiles), 1 << 24));
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        row[i] = plan_row<RT, CLASSES>(mine[i], G, nkv, Q);
        sum.units += row[i].units;
        sum.few += row[i].few;
        sum.split += row[i].split;
        sum.part += row[i].part;
    }
    bool last;
    if (!place<SPLIT, SORT>(SPLIT ? 0 : wave_total(sum.units), SORT ? wave_total(sum.few) : 0, SPLIT ? wave_total(sum.split) : 0, u, last))
        return false;
    const int c = counted<SPLIT>(sum, last), s = wave_scan(c);
    const uint64_t past = __ballot(s > u);
    if (past == 0) return false;
    const int l = __builtin_ctzll(past);
    u -= __builtin_amdgcn_readlane(s - c, l);
    part = wave_total(lane < l ? sum.part : 0);
    un.b = PER * l;
    un.sq = lane_seq(mine[0], l);
#pragma unroll
    for (int i = 0; i + 1 < PER; ++i) {                  // among the lane's sequences
        const int ci = __builtin_amdgcn_readlane(counted<SPLIT>(row[i], last), l);
        if (u < ci) break;
        u -= ci;
        part += __builtin_amdgcn_readlane(row[i].part, l);
        un.b = PER * l + i + 1;
        un.sq = lane_seq(mine[i + 1], l);
    }
    return true;
}

// The workgroup's unit, or false if it has none.  SPLIT: its split tile instead, as the tile's first piece.
template <int RT, bool SPLIT, bool SORT>
__device__ __forceinline__ bool find_unit(const AttnChunkArgs& a, int G, Unit& un) {
    const int nkv = a.kv.n_kv_heads, n_seqs = a.chunk.n_seqs;
    int Q, u, part;
    if (__builtin_expect(n_seqs <= 64, 1)) {
        if (!find_by_lanes<RT, SPLIT, SORT, 1>(a, G, un, Q, u, part)) return false;
    } else if (n_seqs <= PLAN_LANES) {
        if (!find_by_lanes<RT, SPLIT, SORT, PER_LANE>(a, G, un, Q, u, part)) return false;
    } else {
        bool last;
        if (!place<SPLIT, SORT>(a.plan[PLAN_UNITS], a.plan[PLAN_FEW], a.plan[PLAN_SPLIT], u, last)) return false;
        const PlanRow* rows = (const PlanRow*)(a.plan + PLAN_HEAD);
        un.b = last_at_most(n_seqs, u, [&](int b) { return counted<SPLIT>(rows[b], last); });
        if (un.b < 0) return false;
        Q = a.plan[PLAN_Q];
        u -= counted<SPLIT>(rows[un.b], last);
        part = rows[un.b].part;
        un.sq = load_seq(a.chunk, un.b);
    }
    const Plan pl = plan_seq<RT>(un.sq, G, Q);
    const int units = SPLIT ? pl.tiles * nkv : pl.tiles * pl.pieces * nkv;
    if (u < 0 || u >= units) return false;             // overlapping rows: sums past int32
    un.pieces = pl.pieces;
    un.rt = u % pl.tiles;
    const int v = u / pl.tiles, sp = SPLIT ? 0 : v % pl.pieces;
    un.kvh = SPLIT ? v : v / pl.pieces;
    un.part = part + (SPLIT ? un.kvh * pl.pieces * pl.tiles + un.rt : u);
    // the blocks up to the tile's last row, in equal pieces
    const int last_row = min((un.rt + 1) * RT, un.sq.n * G) - 1;
    const int blocks = min(pl.blocks, (un.sq.ctx + last_row / G) / VT_BLK + 1), per = (blocks + pl.pieces - 1) / pl.pieces;
    un.beg = sp * per;
    un.end = min(un.beg + per, blocks);
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

// Where a piece of a 256-row tile keeps dims d0 .. d0 + 3 of row r: the accumulators as the lanes hold them (whole
// kilobytes); (m, l) of row r at TILE_ROWS D + 2 r.
template <int D>
__device__ __forceinline__ int tile_part(int r, int d0) {
    return ((r >> 5) * (D / 8) + (d0 >> 3)) * 256 + 4 * ((r & 31) + 8 * (d0 & 4));
}

}  // namespace fpk
