// A unit of the chunk attention with few rows: a wave's blocks stream through its registers, keys first, values
// behind them.  (attn_chunk.hip has the method and what it measured.)
#pragma once
#include <type_traits>

#include "attn_plan.h"

namespace fpk {

// The largest v of the lanes with this lane's column (l % 16): in registers, where a shuffle goes through LDS.
__device__ __forceinline__ float max_groups(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The softmax's reference moves only when a score passes it by 2^SLACK, so that few blocks rescale the sums.
// bf16 caches: and then to 2^(SLACK + ROOM) above that score, so that probabilities are at most 2^-ROOM and values up to
// 2^127 cannot overflow the sums of 2^24 positions (bf16 and fp32 have exponents enough below).
constexpr float SLACK = 8.f, ROOM = 24.f;

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

// LDS of a unit of 16 NT rows
template <int D, int NT>
struct StreamLds {
    static constexpr int RT = 16 * NT, RS = D + 4;
    __attribute__((aligned(16))) float ow[4][RT * RS];
    float mw[4][RT], lw[4][RT];
    int sw[4];
};

// One unit of at most 16 NT rows.  TILE: its partial result is laid out as those of the 256-row tiles.
template <int D, bool KV8, int NT, bool TILE>
__device__ __forceinline__ void stream_unit(const AttnChunkArgs& a, const Unit& un, StreamLds<D, NT>& lds) {
    constexpr int NJ = D / 32, ND = D / 16, RT = 16 * NT;
    constexpr int NK = Chunk<D, KV8>::NK;
    constexpr int RS = D + 4;
    auto& ow = lds.ow;
    auto& mw = lds.mw;
    auto& lw = lds.lw;
    auto& sw = lds.sw;
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r = lane & 15, g = lane >> 4;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
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
    constexpr int KB = VT_BLK * D * (KV8 ? 1 : 2);      // bytes of a block of keys, and of values
    Chunk<D, KV8> c;
    auto load_k = [&](int i) {
        const int pb = __builtin_amdgcn_readlane(pbs, i & 63);
        const bool ok = pb >= 0;
        const int64_t at = ok ? pb : 0;
        const auto rk = buf_rsrc((const char*)a.kv.k + at * KB, ok ? KB : 0);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < NK; ++x)
                c.k[t][x] = __builtin_amdgcn_raw_buffer_load_b128(rk, (16 * t + r) * D * (KV8 ? 1 : 2) + 64 * x + 16 * g, 0, 0);
        if constexpr (KV8) {
            const auto sk = buf_rsrc(a.kv.k_scales + at * VT_BLK, ok ? 2 * VT_BLK : 0);
#pragma unroll
            for (int t = 0; t < 2; ++t) c.ks[t] = __builtin_amdgcn_raw_buffer_load_b64(sk, (16 * t + 4 * g) * 2, 0, 0);
        }
    };
    auto load_v = [&](int i) {
        const int pb = __builtin_amdgcn_readlane(pbs, i & 63);
        const bool ok = pb >= 0;
        const int64_t at = ok ? pb : 0;
        const auto rv = buf_rsrc((const char*)a.kv.v + at * KB, ok ? KB : 0);
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) {
            const int off = ((16 * dd + r) * VT_BLK + 8 * g) * (KV8 ? 1 : 2);
            if constexpr (KV8) c.v[dd] = __builtin_amdgcn_raw_buffer_load_b64(rv, off, 0, 0);
            else c.v[dd] = __builtin_amdgcn_raw_buffer_load_b128(rv, off, 0, 0);
        }
        if constexpr (KV8) {
            const auto sv = buf_rsrc(a.kv.v_scales + at * VT_BLK, ok ? 2 * VT_BLK : 0);
#pragma unroll
            for (int t = 0; t < 2; ++t) c.vs[t] = __builtin_amdgcn_raw_buffer_load_b64(sv, (16 * t + 4 * g) * 2, 0, 0);
        }
    };
    if (n > 0) {
        load_k(0);
        load_v(0);
    }

    // queries: column c of tile t is row row0 + 16 t + c.  Columns past the last row see no position, so
    // what they hold does not matter.
    u32x4 qf[NT][NJ];
    int lim[NT];                                 // last position that the lane's row sees
    const QScale qs = q_scale(a.scale);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int rho = row0 + 16 * t + r;
        const bool live = 16 * t + r < rows;
        const int tok = live ? rho / G : 0, h = live ? rho % G : 0;
        lim[t] = live ? sq.ctx + tok : -1;
        const uint16_t* q = a.q + (int64_t)(sq.row0 + tok) * a.q_stride + (kvh * G + h) * D;
#pragma unroll
        for (int j = 0; j < NJ; ++j) qf[t][j] = (*(const u32x4*)(q + qdim<KV8>(j, g)) ^ qs.sign) & qs.keep;
    }

    f32x4 oacc[NT][ND];
    float m_run[NT], l_run[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        m_run[t] = -INFINITY;
        l_run[t] = 0.f;
#pragma unroll
        for (int dd = 0; dd < ND; ++dd) oacc[t][dd] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float sl2 = qs.sl2;

    bool strays = false;
    // Block i from c, which is refilled with block `next`, keys and values as soon as they are used.  (A second
    // buffer would cost a third of the waves, and its second copy of this code as much again in instruction fetch where a
    // wave has few blocks: one sequence of 331 on 32 kv heads 10.6 us instead of 9.5, 200 of up to 600 221 instead of 194;
    // only long bf16 batches, bound by memory, gain 2 %.)
    auto compute = [&](int i, int next) {
        const int base = (beg + w + 4 * i) * VT_BLK;
        float ksc[2][4], vsc[2][4], lk = SLACK + ROOM;       // lk: from the block's largest score to its reference
        const bool edge = base + VT_BLK > sq.ctx + 1;        // some row may not see all of the block
        // positions past the sequence hold anything: their values must not meet a zero probability (cleared before the
        // look for values that are not finite, which would take them for the sequence's)
        if (base + VT_BLK > sq.len) {
            const int nk = sq.len - base;
            if constexpr (KV8) {
#pragma unroll
                for (int t = 0; t < 2; ++t) c.vs[t] &= u32x2{slots_below(g, 2 * t, nk), slots_below(g, 2 * t + 1, nk)};
            } else {
#pragma unroll
                for (int dd = 0; dd < ND; ++dd)
#pragma unroll
                    for (int x = 0; x < 4; ++x) c.v[dd][x] &= slots_below(g, x, nk);
            }
        }
        if (edge) {
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
        // P v_scale is at most 2^15: log2 of the block's largest value scale, less 15 and the reference's
        // slack.  Products down to 2^-21 of the largest keep fp16's full precision.
        if constexpr (KV8) {
            float m = 5.9604645e-8f;             // 2^-24, the least fp16
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(vsc[t][e]));
            m = max_groups(m);
            lk = __builtin_amdgcn_logf(fminf(m, 65504.f)) - (15.f - SLACK);
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
        bool grown = false;
#pragma unroll
        for (int q = 0; q < NT; ++q) {
            float s[2][4];                       // scores; int8: to base 2 already
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NJ; ++j) acc = mfma_bf16(kf[t][j], qf[q][j], acc);
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][e] = KV8 ? acc[e] * ksc[t][e] : acc[e];
            }
            if (edge) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][e] = base + 16 * t + 4 * g + e <= lim[q] ? s[t][e] : -INFINITY;
            }
            float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                             fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            mx = max_groups(mx) * (KV8 ? 1.f : sl2) + lk;
            const float m_new = mx > m_run[q] + SLACK ? mx : m_run[q];
            const float ms = m_new == -INFINITY ? 0.f : m_new;        // nothing seen yet: all zero
            al[q] = __builtin_amdgcn_exp2f(m_run[q] - ms);
            grown |= al[q] != 1.f;
            m_run[q] = m_new;
            float ps = 0.f;
            uint32_t pw[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(KV8 ? s[t][e] - ms : fmaf(s[t][e], sl2, -ms));
                    ps += p[e];
                    if constexpr (KV8) p[e] *= vsc[t][e];
                }
                pw[2 * t] = KV8 ? pack_f16_hw(p[0], p[1]) : pack_bf16_hw(p[0], p[1]);
                pw[2 * t + 1] = KV8 ? pack_f16_hw(p[2], p[3]) : pack_bf16_hw(p[2], p[3]);
            }
            l_run[q] = l_run[q] * al[q] + ps;     // this lane's keys; the lane groups join at the end
            pf[q] = u32x4{pw[0], pw[1], pw[2], pw[3]};
        }
        load_k(next);
        if (__ballot(grown) != 0) {
#pragma unroll
            for (int q = 0; q < NT; ++q)
#pragma unroll
                for (int dd = 0; dd < ND; ++dd) oacc[q][dd] *= al[q];
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
            for (int q = 0; q < NT; ++q) oacc[q][dd] = mfma16<KV8 ? ACT_F16 : ACT_BF16>(vf, pf[q], oacc[q][dd]);
        }
        load_v(next);
    };

    if (n > 0) {
        // past the last the loads fetch it again, so that every trip issues the same number
        for (int i = 0; i < n; ++i) {
            if (((i + 1) & 63) == 0 && i + 1 < n) pages(i + 1);
            compute(i, min(i + 1, n - 1));
        }
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
            const f32x2 ml = f32x2{fmaxf(m, M0), l};
            if constexpr (TILE) {
                float* dst = a.ws + (int64_t)un.part * TILE_ROWS * wst(D);
                *(f32x4*)(dst + tile_part<D>(c, d0)) = o;
                if (d0 == 0) *(f32x2*)(dst + TILE_ROWS * D + 2 * c) = ml;
            } else {
                float* dst = a.ws + ((int64_t)un.part * RT + c) * wst(D);
                *(f32x4*)(dst + d0) = o;
                if (d0 == 0) *(f32x2*)(dst + D) = ml;
            }
        }
    }
}

}  // namespace fpk
