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

#include <type_traits>

#include "attn_plan.h"

namespace fpk {

namespace {

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
__global__ void __launch_bounds__(256, NT == 4 ? 1 : 2) attn_chunk_kernel(AttnChunkArgs a) {
    constexpr int NJ = D / 32, ND = D / 16, RT = 16 * NT;
    constexpr int NK = Chunk<D, KV8>::NK;
    constexpr int RS = D + 4;
    __shared__ __attribute__((aligned(16))) float ow[4][RT * RS];
    __shared__ float mw[4][RT], lw[4][RT];
    __shared__ int sw[4];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<false, false>(a, G, RT, un)) return;
    const Seq& sq = un.sq;
    const int b = un.b, kvh = un.kvh, beg = un.beg, end = un.end;
    const int row0 = un.rt * RT, rows = min(RT, sq.n * G - row0);

    // the pool block of this wave's i-th block, 64 of them at a time in the lanes
    const int n = end > beg ? (end - beg - w + 3) / 4 : 0;
    int pbs = 0;
    auto pages = [&](int i0) {
        const int i = i0 + lane;
        pbs = i < n ? pool_block(a.kv, a.chunk, b, kvh, beg + w + 4 * i) : -1;
    };
    pages(0);                                   // on its way while the queries are addressed
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

    bool strays = false;
    auto compute = [&](int i, Chunk<D, KV8>& c) {
        const int base = (beg + w + 4 * i) * VT_BLK;
        float ksc[2][4], vsc[2][4], lk = 0.f;
        if (base + VT_BLK > sq.ctx + 1) {        // some row may not see all of the block
            uint32_t bad = 0;
            if constexpr (KV8) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    bad |= nonfinite<F16_EXP>(c.vs[t].x) | nonfinite<F16_EXP>(c.vs[t].y);
                    c.vs[t] = u32x2{finite_halves<F16_EXP>(c.vs[t].x), finite_halves<F16_EXP>(c.vs[t].y)};
                }
            } else {
#pragma unroll
                for (int dd = 0; dd < ND; ++dd)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        bad |= nonfinite<BF16_EXP>(c.v[dd][x]);
                        c.v[dd][x] = finite_halves<BF16_EXP>(c.v[dd][x]);
                    }
            }
            strays |= __ballot(bad != 0) != 0;
        }
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
#pragma unroll
                    for (int x = 0; x < 4; ++x) c.v[dd][x] &= slots_below(g, x, nk);
                }
            }
            if constexpr (KV8) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) vsc[t][e] = 16 * t + 4 * g + e < nk ? vsc[t][e] : 0.f;
            }
        }
        // P v_scale is at most 2^15: log2 of the block's largest value scale, less 15.  Products down to
        // 2^-29 of the largest keep fp16's full precision.
        if constexpr (KV8) {
            float m = 5.9604645e-8f;             // 2^-24, the least fp16
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(vsc[t][e]));
            m = fmaxf(m, __shfl_xor(m, 16, 64));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            lk = __builtin_amdgcn_logf(fminf(m, 65504.f)) - 15.f;
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
            const float m_new = fmaxf(m_run[q], mx + lk);
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
                pw[2 * t] = KV8 ? pack_f16_hw(p[0], p[1]) : pack_bf16_hw(p[0], p[1]);
                pw[2 * t + 1] = KV8 ? pack_f16_hw(p[2], p[3]) : pack_bf16_hw(p[2], p[3]);
            }
            l_run[q] = l_run[q] * al[q] + ps;     // this lane's keys; the lane groups join at the end
            pf[q] = u32x4{pw[0], pw[1], pw[2], pw[3]};
        }
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) {
            u32x4 vf;
            if constexpr (KV8) {
                const u32x2 c0 = i8x4_to_f16x4(c.v[dd].x), c1 = i8x4_to_f16x4(c.v[dd].y);
                vf = u32x4{c0.x, c0.y, c1.x, c1.y};
            } else {
                vf = c.v[dd];
            }
#pragma unroll
            for (int q = 0; q < NT; ++q) {
                oacc[q][dd] *= al[q];
                oacc[q][dd] = mfma16<KV8 ? ACT_F16 : ACT_BF16>(vf, pf[q], oacc[q][dd]);
            }
        }
    };

    if (n > 0) {
        // two blocks in flight; past the last the loads fetch it again, so that every trip issues
        // the same number
        Chunk<D, KV8> ca, cb;
        load(0, ca);
        load(min(1, n - 1), cb);
        int i = 0;
        for (; i + 2 <= n; i += 2) {
            if (((i + 2) & 63) == 0 && i + 2 < n) pages(i + 2);
            compute(i, ca);
            load(min(i + 2, n - 1), ca);
            compute(i + 1, cb);
            load(min(i + 3, n - 1), cb);
        }
        if (i < n) compute(i, ca);
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
    if (lane == 0) sw[w] = strays;
    // merge the four waves
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) *(f32x4*)(&ow[w][(16 * t + r) * RS + 16 * dd + 4 * g]) = oacc[t][dd];
    __syncthreads();
#pragma unroll 4
    for (int it = tid; it < rows * (D / 4); it += 256) {
        const int c = it / (D / 4), d0 = it % (D / 4) * 4;
        float m = -INFINITY;
#pragma unroll
        for (int v = 0; v < 4; ++v) m = fmaxf(m, mw[v][c]);
        float l = 0.f;
        f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float mv = mw[v][c];
            const float e = mv == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mv - m);
            l += lw[v][c] * e;
            o += *(const f32x4*)&ow[v][c * RS + d0] * e;
        }
        const int rho = row0 + c;
        if (sw[0] | sw[1] | sw[2] | sw[3]) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                const float x = stray_sum<D, KV8>(a, b, kvh, d0 + e, max(beg, (sq.ctx + 1) / VT_BLK) * VT_BLK,
                                                  min(sq.ctx + rho / G, end * VT_BLK - 1));
                o += f32x4{e == 0 ? x : 0.f, e == 1 ? x : 0.f, e == 2 ? x : 0.f, e == 3 ? x : 0.f};
            }
        }
        if (un.pieces == 1) {
            store4(a.out + ((int64_t)(sq.row0 + rho / G) * a.n_heads + kvh * G + rho % G) * D + d0, o * (1.f / l), a.out_fmt);
        } else {
            float* dst = a.ws + ((int64_t)un.part * RT + c) * wst(D);
            *(f32x4*)(dst + d0) = o;
            if (d0 == 0) {
                dst[D] = m;
                dst[D + 1] = l;
            }
        }
    }
}

// Joins the pieces of split tiles: RPW rows of a tile per workgroup, a thread per four dims of a row.
// Pieces' statistics and outputs load eight at a time.
template <int D, int RT>
__global__ void __launch_bounds__(256) attn_chunk_join_kernel(AttnChunkArgs a) {
    constexpr int RPW = 1024 / D, NS = RT / RPW;         // rows per workgroup; workgroups per tile
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<true, false>(a, G, RT, un)) return;
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

// log2 of the pieces a call aims for, and the least number of blocks worth a piece
int piece_target(int RT) { return RT >= 64 ? 8 : 10; }
int piece_min(int RT) { return RT == TILE_ROWS ? 8 : 16; }

}  // namespace

// Split tiles have more than Q blocks, so their pieces number at most twice total / Q, twice the aim.
size_t attn_chunk_ws_bytes(const fp_paged_kv& kv, const fp_chunk& c, int n_heads) {
    const int RT = tile_rows(c, n_heads / kv.n_kv_heads);
    return ((size_t)2 << piece_target(RT)) * RT * wst(kv.head_dim) * sizeof(float);
}

template <int D, bool KV8, int RT>
static hipError_t launch_rt(AttnChunkArgs a, hipStream_t st) {
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    const int64_t tiles = std::min<int64_t>((int64_t)a.chunk.n_rows * G, (int64_t)a.chunk.n_rows * G / RT + a.chunk.n_seqs) * nkv;
    a.target = piece_target(RT);
    a.min_blocks = piece_min(RT);
    // tiles of 64 rows and more: one workgroup per CU
    a.slots = RT >= 64 ? 8 : 0;
    a.over = 10;
    a.join = 8;
    const int64_t pieces = (int64_t)1 << a.target, n = std::max(tiles + pieces, 2 * pieces) + 8;
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
