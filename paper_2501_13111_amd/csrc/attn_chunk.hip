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

#include "paged.h"

namespace fpk {

namespace {

// pieces a call aims for: enough waves to keep every CU's loads in flight
constexpr int TARGET = 768;
constexpr int MINB = 16;                   // blocks per piece at least: four per wave

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
// Blocks per piece: from the total over all sequences.
__device__ __forceinline__ int plan_q(const AttnChunkArgs& a, int G, int RT) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int b = lane; b < a.chunk.n_seqs; b += 64) {
        const Seq s = load_seq(a.chunk, b);
        const Plan p = plan_seq(s, G, RT, 1);
        total += (int64_t)p.tiles * p.blocks;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o, 64);
    total = (total * a.kv.n_kv_heads + a.target - 1) / a.target;
    return (int)std::max<int64_t>(a.min_blocks, std::min<int64_t>(total, 1 << 24));
}

constexpr int wst(int D) { return D + 4; }     // floats per row of a piece: o, then m, l

template <int D, bool KV8>
struct Chunk {
    static constexpr int NK = KV8 ? D / 64 : D / 32;   // 16-byte key loads per 16-key tile
    u32x4 k[2][NK];
    typename std::conditional<KV8, u32x2, u32x4>::type v[D / 16];
    u32x2 ks[2], vs[2];
};

// dims that k-step j of lane group g covers (the queries take the same order)
template <bool KV8>
__device__ __forceinline__ int qdim(int j, int g) {
    return KV8 ? 64 * (j >> 1) + 16 * g + 8 * (j & 1) : 32 * j + 8 * g;
}

// Eight int8 codes -> bf16 (exact).
__device__ __forceinline__ u32x4 i8x8_to_bf16(uint32_t lo, uint32_t hi) {
    auto two = [](uint32_t w, int s) {
        const uint32_t a = __float_as_uint((float)(int8_t)(w >> s)), b = __float_as_uint((float)(int8_t)(w >> (s + 8)));
        return __builtin_amdgcn_perm(b, a, 0x07060302u);
    };
    return u32x4{two(lo, 0), two(lo, 16), two(hi, 0), two(hi, 16)};
}

template <int D, bool KV8, int NT>
__global__ void __launch_bounds__(256, 2) attn_chunk_kernel(AttnChunkArgs a) {
    constexpr int NJ = D / 32, ND = D / 16, RT = 16 * NT;
    constexpr int NK = Chunk<D, KV8>::NK;
    constexpr int RS = D + 4;
    __shared__ __attribute__((aligned(16))) float ow[4][16 * RS];
    __shared__ float mw[4][RT], lw[4][RT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    const int Q = plan_q(a, G, RT);
    int u = blockIdx.x, part = 0;                // part: pieces of split tiles before this one
    int b = -1;
    {
        int u2 = u;
        b = find_seq(a.chunk.n_seqs, u2, [&](int i) {
            const Plan p = plan_seq(load_seq(a.chunk, i), G, RT, Q);
            return p.tiles * p.pieces * nkv;
        });
        if (b < 0) return;
        // split pieces of the sequences before b
        for (int i = lane; i < b; i += 64) {
            const Plan p = plan_seq(load_seq(a.chunk, i), G, RT, Q);
            if (p.pieces > 1) part += p.tiles * p.pieces * nkv;
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) part += __shfl_xor(part, o, 64);
        u = u2;
    }
    const Seq sq = load_seq(a.chunk, b);
    const Plan pl = plan_seq(sq, G, RT, Q);
    if (u < 0 || u >= pl.tiles * pl.pieces * nkv) return;      // overlapping rows: sums past int32
    part += u;
    // piece -> (kv head, piece of the keys, row tile)
    const int rt = u % pl.tiles, sp = u / pl.tiles % pl.pieces, kvh = u / (pl.tiles * pl.pieces);
    const int row0 = rt * RT, rows = min(RT, sq.n * G - row0);
    // blocks: the piece's share, no further than the tile's last row sees
    const int tblocks = (sq.ctx + (row0 + rows - 1) / G) / VT_BLK + 1;
    const int per = (pl.blocks + pl.pieces - 1) / pl.pieces;
    const int beg = sp * per, end = min(min(beg + per, pl.blocks), tblocks);

    // queries: column c of tile t is row row0 + 16 t + c
    u32x4 qf[NT][NJ];
    int lim[NT];                                 // last position that the lane's row sees
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int rho = row0 + 16 * t + r;
        const bool live = 16 * t + r < rows;
        const int tok = live ? rho / G : 0, h = live ? rho % G : 0;
        lim[t] = live ? sq.ctx + tok : -1;
        const uint16_t* q = a.q + (int64_t)(sq.row0 + tok) * a.q_stride + (kvh * G + h) * D;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const u32x4 x = *(const u32x4*)(q + qdim<KV8>(j, g));
            qf[t][j] = live ? x : u32x4{0u, 0u, 0u, 0u};
        }
    }

    // the pool block of this wave's i-th block, 64 of them at a time in the lanes
    const int n = end > beg ? (end - beg - w + 3) / 4 : 0;
    int pbs = 0;
    auto pages = [&](int i0) {
        const int i = i0 + lane;
        pbs = i < n ? pool_block(a.kv, a.chunk, b, kvh, beg + w + 4 * i) : -1;
    };
    constexpr int KB = VT_BLK * D * (KV8 ? 1 : 2);      // bytes of a block of keys, and of values
    auto load = [&](int i, Chunk<D, KV8>& c) {
        const int pb = __builtin_amdgcn_readlane(pbs, i & 63);
        const bool ok = pb >= 0;
        const int64_t at = ok ? pb : 0;
        const auto rk = buf_rsrc((const char*)a.kv.k + at * KB, ok ? KB : 0);
        const auto rv = buf_rsrc((const char*)a.kv.v + at * KB, ok ? KB : 0);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < NK; ++x)
                c.k[t][x] = __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * t + r) * D * (KV8 ? 1 : 2) + 64 * x + 16 * g, 0, 0);
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) {
            const int off = ((16 * dd + r) * VT_BLK + 8 * g) * (KV8 ? 1 : 2);
            if constexpr (KV8) c.v[dd] = __builtin_amdgcn_raw_buffer_load_b64(rv, off, 0, 0);
            else c.v[dd] = __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0);
        }
        if constexpr (KV8) {
            const auto sk = buf_rsrc(a.kv.k_scales + at * VT_BLK, ok ? 2 * VT_BLK : 0);
            const auto sv = buf_rsrc(a.kv.v_scales + at * VT_BLK, ok ? 2 * VT_BLK : 0);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                c.ks[t] = __builtin_amdgcn_raw_buffer_load_b64(sk, (16 * t + 4 * g) * 2, 0, 0);
                c.vs[t] = __builtin_amdgcn_raw_buffer_load_b64(sv, (16 * t + 4 * g) * 2, 0, 0);
            }
        }
    };

    f32x4 oacc[NT][ND];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = -INFINITY;
        l_run[t] = 0.f;
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) oacc[t][dd] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float sl2 = a.scale * 1.4426950408889634f;

    auto compute = [&](int i, Chunk<D, KV8>& c) {
        const int base = (beg + w + 4 * i) * VT_BLK;
        float ksc[2][4], vsc[2][4];
        if constexpr (KV8) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ksc[t][e] = h2f((uint16_t)((e < 2 ? c.ks[t].x : c.ks[t].y) >> (16 * (e & 1)))) * sl2;
                    vsc[t][e] = h2f((uint16_t)((e < 2 ? c.vs[t].x : c.vs[t].y) >> (16 * (e & 1))));
                }
        }
        // positions past the sequence hold anything: their values must not meet a zero probability
        if (base + VT_BLK > sq.len) {
            const int nk = sq.len - base;
#pragma unroll
            for (int dd = 0; dd < ND; ++dd) {
                if constexpr (!KV8) {
                    u32x4 m;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {        // word x: slots 8 g + 2 x, + 1: keys 16 (x / 2) + 4 g + 2 (x % 2), + 1
                        const int key = 16 * (x >> 1) + 4 * g + 2 * (x & 1);
                        m[x] = (key < nk ? 0x0000FFFFu : 0u) | (key + 1 < nk ? 0xFFFF0000u : 0u);
                    }
                    c.v[dd] &= m;
                }
            }
            if constexpr (KV8) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) vsc[t][e] = 16 * t + 4 * g + e < nk ? vsc[t][e] : 0.f;
            }
        }
        u32x4 kf[2][NJ];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if constexpr (KV8) {
                    const u32x4 x = c.k[t][j >> 1];
                    kf[t][j] = (j & 1) ? i8x8_to_bf16(x.z, x.w) : i8x8_to_bf16(x.x, x.y);
                } else {
                    kf[t][j] = c.k[t][j];
                }
            }
        u32x4 pf[NT];
        float al[NT];
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            float s[2][4];
            float mx = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc = mfma_bf16(kf[t][j], qf[q][j], acc);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = KV8 ? acc[e] * ksc[t][e] : acc[e] * sl2;
                    s[t][e] = base + 16 * t + 4 * g + e <= lim[q] ? v : -INFINITY;
                    mx = fmaxf(mx, s[t][e]);
                }
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m_run[q], mx);
            const float ms = m_new == -INFINITY ? 0.f : m_new;        // nothing seen yet: all zero
            al[q] = __builtin_amdgcn_exp2f(m_run[q] - ms);
            m_run[q] = m_new;
            float ps = 0.f;
            uint32_t pw[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(s[t][e] - ms);
                    ps += p[e];
                    if constexpr (KV8) p[e] *= vsc[t][e];
                }
                pw[2 * t] = pack_bf16_hw(p[0], p[1]);
                pw[2 * t + 1] = pack_bf16_hw(p[2], p[3]);
            }
            l_run[q] = l_run[q] * al[q] + ps;     // this lane's keys; the lane groups join at the end
            pf[q] = u32x4{pw[0], pw[1], pw[2], pw[3]};
        }
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) {
            u32x4 vf;
            if constexpr (KV8) vf = i8x8_to_bf16(c.v[dd].x, c.v[dd].y);
            else vf = c.v[dd];
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                oacc[q][dd] *= al[q];
                oacc[q][dd] = mfma_bf16(vf, pf[q], oacc[q][dd]);
            }
        }
    };

    for (int i = 0; i < n; ++i) {
        if ((i & 63) == 0) pages(i);
        Chunk<D, KV8> c;
        load(i, c);
        compute(i, c);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        l_run[t] += __shfl_xor(l_run[t], 16, 64);
        l_run[t] += __shfl_xor(l_run[t], 32, 64);
        if (g == 0) {
            mw[w][16 * t + r] = m_run[t];
            lw[w][16 * t + r] = l_run[t];
        }
    }
    // merge the four waves, one tile of 16 rows after another
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        __syncthreads();
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) *(f32x4*)(&ow[w][r * RS + 16 * dd + 4 * g]) = oacc[t][dd];
        __syncthreads();
        for (int it = tid; it < 16 * (D / 4); it += 256) {
            const int c = it / (D / 4), d0 = it % (D / 4) * 4;
            if (16 * t + c >= rows) continue;
            float m = -INFINITY;
#pragma unroll
            for (int v = 0; v < 4; ++v) m = fmaxf(m, mw[v][16 * t + c]);
            float l = 0.f;
            f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float mv = mw[v][16 * t + c];
                const float e = mv == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv - m);
                l += lw[v][16 * t + c] * e;
                o += *(const f32x4*)&ow[v][c * RS + d0] * e;
            }
            const int rho = row0 + 16 * t + c;
            if (pl.pieces == 1) {
                const float inv = 1.f / l;
                uint16_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = act_store((float)(__bf16)(o[e] * inv), a.out_fmt);
                *(u32x2*)(a.out + ((int64_t)(sq.row0 + rho / G) * a.n_heads + kvh * G + rho % G) * D + d0) =
                    u32x2{(uint32_t)x[0] | ((uint32_t)x[1] << 16), (uint32_t)x[2] | ((uint32_t)x[3] << 16)};
            } else {
                float* dst = a.ws + ((int64_t)part * RT + 16 * t + c) * wst(D);
                *(f32x4*)(dst + d0) = o;
                if (d0 == 0) {
                    dst[D] = m;
                    dst[D + 1] = l;
                }
            }
        }
    }
}

// Joins the pieces of split tiles: a workgroup per (sequence, kv head, row tile), a thread per
// four dims of a row.
template <int D, int NT>
__global__ void __launch_bounds__(256) attn_chunk_join_kernel(AttnChunkArgs a) {
    constexpr int RT = 16 * NT;
    const int lane = threadIdx.x & 63;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    const int Q = plan_q(a, G, RT);
    int u = blockIdx.x;
    const int b = find_seq(a.chunk.n_seqs, u, [&](int i) {
        const Plan p = plan_seq(load_seq(a.chunk, i), G, RT, Q);
        return p.pieces > 1 ? p.tiles * nkv : 0;
    });
    if (b < 0) return;
    int part = 0;
    for (int i = lane; i < b; i += 64) {
        const Plan p = plan_seq(load_seq(a.chunk, i), G, RT, Q);
        if (p.pieces > 1) part += p.tiles * p.pieces * nkv;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) part += __shfl_xor(part, o, 64);
    const Seq sq = load_seq(a.chunk, b);
    const Plan pl = plan_seq(sq, G, RT, Q);
    if (u < 0 || u >= pl.tiles * nkv) return;
    const int rt = u % pl.tiles, kvh = u / pl.tiles;
    const int row0 = rt * RT, rows = min(RT, sq.n * G - row0);
    part += kvh * pl.tiles * pl.pieces + rt;
    for (int it = threadIdx.x; it < rows * (D / 4); it += 256) {
        const int c = it / (D / 4), d0 = it % (D / 4) * 4;
        const float* src = a.ws + ((int64_t)part * RT + c) * wst(D);
        const int64_t step = (int64_t)pl.tiles * RT * wst(D);
        float m = -INFINITY;
        for (int i = 0; i < pl.pieces; ++i) m = fmaxf(m, src[i * step + D]);
        float l = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int i = 0; i < pl.pieces; ++i) {
            const float mi = src[i * step + D];
            const float e = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mi - m);
            l += src[i * step + D + 1] * e;
            o += *(const f32x4*)(src + i * step + d0) * e;
        }
        const int rho = row0 + c;
        const float inv = 1.f / l;
        uint16_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = act_store((float)(__bf16)(o[e] * inv), a.out_fmt);
        *(u32x2*)(a.out + ((int64_t)(sq.row0 + rho / G) * a.n_heads + kvh * G + rho % G) * D + d0) =
            u32x2{(uint32_t)x[0] | ((uint32_t)x[1] << 16), (uint32_t)x[2] | ((uint32_t)x[3] << 16)};
    }
}

int row_tiles(const fp_chunk& c, int G) {
    const int64_t R = std::min<int64_t>((int64_t)c.max_new * G, 1 << 20);
    return R <= 16 ? 1 : R <= 32 ? 2 : 4;
}

}  // namespace

// Split tiles have more than Q blocks, so their pieces number at most twice total / Q, twice the target.
size_t attn_chunk_ws_bytes(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    const int RT = 16 * row_tiles(c, n_heads / kv.n_kv_heads);
    return (size_t)2 * TARGET * RT * wst(kv.head_dim) * sizeof(float);
}

template <int D, bool KV8, int NT>
static hipError_t launch_nt(AttnChunkArgs a, hipStream_t st) {
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    const int64_t tiles = std::min<int64_t>((int64_t)a.chunk.n_rows * G, (int64_t)a.chunk.n_rows * G / (16 * NT) + a.chunk.n_seqs) * nkv;
    const int64_t n = tiles + TARGET;
    if (n > INT_MAX) return hipErrorInvalidValue;
    a.target = TARGET;
    a.min_blocks = MINB;
    FP_LAUNCH((attn_chunk_kernel<D, KV8, NT>), dim3((unsigned)n), dim3(256), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || (a.chunk.max_len + VT_BLK - 1) / VT_BLK <= MINB) return e;
    // tiles that can be split: each has a piece of at least half of Q blocks
    FP_LAUNCH((attn_chunk_join_kernel<D, NT>), dim3((unsigned)std::min<int64_t>(tiles, TARGET)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <int D, bool KV8>
static hipError_t launch_d(const AttnChunkArgs& a, hipStream_t st) {
    switch (row_tiles(a.chunk, a.n_heads / a.kv.n_kv_heads)) {
        case 1: return launch_nt<D, KV8, 1>(a, st);
        case 2: return launch_nt<D, KV8, 2>(a, st);
        default: return launch_nt<D, KV8, 4>(a, st);
    }
}

hipError_t launch_attn_chunk(const AttnChunkArgs& a, hipStream_t st) {
    const bool i8 = a.kv.format == FP_KV_INT8;
    if (a.kv.head_dim == 128) return i8 ? launch_d<128, true>(a, st) : launch_d<128, false>(a, st);
    if (a.kv.head_dim == 64) return i8 ? launch_d<64, true>(a, st) : launch_d<64, false>(a, st);
    return hipErrorInvalidValue;
}

}  // namespace fpk
