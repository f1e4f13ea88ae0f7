// Attention of drafted trees that bring 65 to 128 rows to a kv head of 128 dims, or more of them over short contexts: tiles of 128 rows,
// eight waves of 32 rows each.
// (Tiles of 256, attn_tile.hip, leave half of their waves without rows; tiles of 64 and 32 read and unpack the cache
// several times.)
//
// Rows, units and the join of their pieces are those of attn_chunk.hip, the mask is the tree's (tree.h).  A step takes two blocks
// of 32 keys: wave w the rows 32 (w % 4) .. and of the two blocks the w / 4-th; the two sums of a row are merged at the end.
//     S^T = K Q^T,   O^T += V^T P^T      on MFMA 32x32x16
// Two waves share a SIMD, w and w + 4: one multiplies first (P V of its last block, then S of this one), stores and takes its softmax, the
// other stores, takes the softmax of its last block and multiplies then.  One barrier a step (with one after each half, the waves
// half a step apart: 32 sequences of 8192, 16 nodes, 64 heads on 8, int8 264 us, so 241; bf16 258 and 253).  Blocks pass
// through registers into LDS, as 16-bit fragments (int8: codes times scales in fp16), loaded two steps before they are stored.
//
// Those 32 sequences with lengths spread up to 8192 (290 MB of int8 cache): 131 to 141 us with the join, by a kernel trace 135 and 10.6.
// Lengths up to 2048, 4096, 16384 and 32768 take 57, 80, 237 and 454; all five fit, within 4 %, 1.3 us a step of two blocks of keys and 9 us a
// unit of prologue and merge, which nothing covers (135 KB of LDS: one workgroup a CU, two units after each other), in the order in
// which the units start: 85 steps on the busiest CU, where an even share is 64.  A step, some 2900 cycles, has 1030 of products on each SIMD, 1300 of LDS
// (a fragment serves the 32 rows of a wave, 128 KB a step, and 32 KB stored) and 200 vector instructions a wave.
#include <type_traits>

#include "attn_stream.h"

namespace fpk {

namespace {

constexpr float LAZY = 8.f;
template <bool KV8>
constexpr float BELOW = KV8 ? 7.f : -(LAZY + ROOM);

constexpr int D = 128, RT = 128, KP = 2;                       // dims, rows of a tile, blocks of a step
constexpr int NKC = D / 16, NDT = D / 32;
constexpr int SB = 2 * NKC * 1024, ST = KP * SB;               // bytes of a block's fragments, and of a step's
constexpr int RS = D + 4;                                      // floats of a row of sums
struct WideLds {
    union {
        __attribute__((aligned(1024))) char ring[3 * ST];
        float ow[KP * RT * RS];
    };
    float mw[KP * RT], lw[KP * RT];
    uint64_t line[TREE_MAX];
    int sw[8];
};

__device__ __forceinline__ uint32_t pk_mul(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) * __builtin_bit_cast(f16x2, y));
}

// v, for code that runs seldom: what is computed from it stays there, and takes no registers in the loop.
__device__ __forceinline__ int rare(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

template <bool KV8>
__global__ void __launch_bounds__(512, 2) attn_wide_kernel(AttnChunkArgs a) {
    constexpr int ES = KV8 ? 1 : 2, KB = VT_BLK * D * ES;
    // A wave loads 1 KB of the pool at a time, of keys or of values: UPB of them make a block, UPW are a wave's of a step.
    constexpr int UPB = 2 * KB / 1024, UPW = KP * UPB / 8, NK = 1024 / (D * ES);
    __shared__ WideLds lds;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<WIDE | RT, false, true>(a, G, un)) return;
    const int row0 = un.rt * RT, rows = min(RT, un.sq.n * G - row0);
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int rg = w % 4, kp = w / 4, l32 = lane & 31, h32 = lane >> 5;
    const Seq& sq = un.sq;
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int b = un.b, kvh = un.kvh, beg = uni(un.beg), n = uni(max(un.end - un.beg, 0)), steps = (n + KP - 1) / KP;

    // the pool blocks of 64 blocks at a time, across the lanes
    int pbs = 0;
    auto pages = [&](int i0) {
        const int i = i0 + lane;
        pbs = i < n ? pool_block(a.kv, a.chunk, b, kvh, beg + i) : -1;
    };
    // Load j of a wave in a step: of block 8 j / UPB.  bf16: even ones are keys, odd ones values; int8: waves 0 to 3 load keys, the others
    // values (`keys`); t: which load of the block's keys or values.  Nothing in a fetch branches: where loads join again the compiler waits for all of them.
    struct Raw {
        u32x4 x[UPW], sa[KV8 ? UPW : 1], sb[KV8 ? UPW : 1];
    };
    const int t = w % (UPB / 2);
    auto fetch = [&](int s, Raw& r, auto keys) {
        if ((s * KP & 63) == 0 && s < steps) pages(s * KP);
#pragma unroll
        for (int j = 0; j < UPW; ++j) {
            const int i = s * KP + 8 * j / UPB;
            const bool key = KV8 ? decltype(keys)::value : j % 2 == 0;
            const int pb = i < n ? __builtin_amdgcn_readlane(pbs, i & 63) : -1;
            const bool ok = pb >= 0;                           // a missing page reads as zeros
            const int64_t at = ok ? pb : 0;
            const auto rs = buf_rsrc((const char*)(key ? a.kv.k : a.kv.v) + at * KB, ok ? KB : 0);
            if constexpr (KV8) {
                // keys: 16 dims of one of 1024 / D keys, and its scale; values: 16 slots of one of 32 dims, and their positions' scales
                const auto sr = buf_rsrc((key ? a.kv.k_scales : a.kv.v_scales) + at * VT_BLK, ok ? 2 * VT_BLK : 0);
                if (key) {
                    const int k = NK * t + lane % NK;
                    r.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rs, k * D + lane / NK * 16, 0, 0);
                    r.sa[j].x = __builtin_amdgcn_raw_buffer_load_b16(sr, 2 * k, 0, 0);
                } else {
                    r.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rs, (32 * t + (lane & 31)) * VT_BLK + (lane >> 5) * 16, 0, 0);
                    r.sa[j] = __builtin_amdgcn_raw_buffer_load_b128(sr, (lane >> 5) * 16, 0, 0);
                    r.sb[j] = __builtin_amdgcn_raw_buffer_load_b128(sr, 32 + (lane >> 5) * 16, 0, 0);
                }
            } else {
                // keys: 8 of them by 8 chunks of 8 dims, the chunks' low bit flipped in every other group; values: 16 dims by 4 chunks of slots
                const int k8 = t & 3;
                r.x[j] = __builtin_amdgcn_raw_buffer_load_b128(rs, key ? (8 * k8 + (lane & 7)) * D * 2 + (8 * (t >> 2) + (lane >> 3 ^ (k8 & 1))) * 16
                                                                       : (16 * t + (lane & 15)) * VT_BLK * 2 + (lane >> 4) * 16, 0, 0);
            }
        }
    };
    // From block `edge` on some node does not see every key: values there that are not finite are taken out (they would make
    // NaN of zero probabilities) and what they are to the rows that do see them is added at the end.  Positions past the
    // sequence hold anything: zeros.  (A step's first block may lie before the edge: its values stay as they are.)
    const int edge = sq.ctx / VT_BLK - beg;
    bool strays = false;
    // LDS layout of a block (attn_tile.hip): keys in groups of 8 by 128 bytes of dims, chunk c of 16 bytes of key k at 1024 (4 (c / 8)
    // + k / 8) + 128 (c % 8, the low bit flipped in every other group) + 16 (k % 8); values 16 dims a group, chunk c (8 slots) of
    // dim d at 1024 (d / 16) + 256 c + 16 (d % 16).  What 8 neighbouring lanes write or read together lies in 128 different bytes.
    auto store = [&](char* slot, int s, const Raw& r, auto keys, auto past_edge) {
#pragma unroll
        for (int j = 0; j < UPW; ++j) {
            const bool key = KV8 ? decltype(keys)::value : j % 2 == 0;
            const bool odd = decltype(past_edge)::value && !key && s * KP + 8 * j / UPB >= edge;
            const int nk = sq.len - (beg + s * KP + 8 * j / UPB) * VT_BLK;
            char* const dst = slot + 8 * j / UPB * SB + (key ? 0 : NKC * 1024);
            uint32_t bad = 0;
            if constexpr (KV8) {
                u32x4 sa = r.sa[j], sb = r.sb[j];
                if (key) {
                    const uint32_t k2 = (sa.x & 0xFFFFu) * 0x10001u;
                    sa = sb = u32x4{k2, k2, k2, k2};
                } else if (odd) {
                    const int c = 2 * (rare(lane) >> 5);
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        sa[x] &= slots_below(c + (x >> 1), x & 1, nk);
                        sb[x] &= slots_below(c + (x >> 1), 2 + (x & 1), nk);
                        bad |= nonfinite<F16_EXP>(sa[x]) | nonfinite<F16_EXP>(sb[x]);
                        sa[x] = finite_halves<F16_EXP>(sa[x]);
                        sb[x] = finite_halves<F16_EXP>(sb[x]);
                    }
                }
                const int k = NK * t + lane % NK, d = 32 * t + (lane & 31);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const u32x2 lo = i8x4_to_f16x4(r.x[j][2 * x]), hi = i8x4_to_f16x4(r.x[j][2 * x + 1]);
                    const int c = 2 * (key ? lane / NK : lane >> 5) + x;
                    const int at = key ? 1024 * (4 * (c >> 3) + (k >> 3)) + 128 * ((c & 7) ^ (k >> 3 & 1)) + 16 * (k & 7)
                                       : 1024 * (d >> 4) + 256 * c + 16 * (d & 15);
                    const u32x4 y = {pk_mul(lo.x, sa[2 * x]), pk_mul(lo.y, sa[2 * x + 1]), pk_mul(hi.x, sb[2 * x]), pk_mul(hi.y, sb[2 * x + 1])};
                    *(u32x4*)(dst + at) = y;
                }
            } else {
                u32x4 y = r.x[j];
                if (odd) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        y[x] &= slots_below(rare(lane) >> 4, x, nk);
                        bad |= nonfinite<BF16_EXP>(y[x]);
                        y[x] = finite_halves<BF16_EXP>(y[x]);
                    }
                }
                *(u32x4*)(dst + t * 1024 + lane * 16) = y;
            }
            if (odd) strays |= __ballot(bad != 0) != 0;
        }
    };
    using Yes = std::integral_constant<bool, true>;
    using No = std::integral_constant<bool, false>;

    // the first loads are on their way while the queries are
    Raw r0, r1;
    if (n > 0) {
        if (!KV8 || w < 4) {
            fetch(0, r0, Yes{});
            fetch(1, r1, Yes{});
        } else {
            fetch(0, r0, No{});
            fetch(1, r1, No{});
        }
    }

    // queries: column l % 32 of the wave's rows; a negative scale turns their signs
    const int rho = row0 + 32 * rg + l32;
    const int wrows = min(max(rows - 32 * rg, 0), 32);
    const bool live = l32 < wrows;
    const int tok = live ? rho / G : 0, h = live ? rho % G : 0;
    uint64_t line = 0;
    {
        uint64_t mine = 0;
        if (un.end * VT_BLK > sq.ctx) mine = tree_lines(a.parent, sq);
        if (w == 0) lds.line[lane] = mine;
        line = __shfl(mine, tok, 64);
    }
    const QScale qs = q_scale(a.scale);
    float sl2 = qs.sl2;
    u32x4 qf[NKC];
    {
        const uint16_t* q = a.q + (int64_t)(sq.row0 + tok) * a.q_stride + (kvh * G + h) * D;
        const uint32_t keep = live ? qs.keep : 0u;
#pragma unroll
        for (int j = 0; j < NKC; ++j) qf[j] = *(const u32x4*)(q + 16 * j + 8 * h32);
        if constexpr (KV8) {
            // fp16, the row's largest to 2^14 .. 2^15 by a power of two that the scale takes back (attn_tile.hip)
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < NKC; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    m = fmaxf(m, fmaxf(fabsf(__uint_as_float(qf[j][x] << 16)), fabsf(__uint_as_float(qf[j][x] & 0xFFFF0000u))));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            const int e = live && m > 0.f ? max(__builtin_amdgcn_frexp_expf(m) - 15, -126) : 0;
            sl2 = fminf(fmaxf(__builtin_amdgcn_ldexpf(sl2, e), 1.2e-38f), 3.4e38f);
            const float f = __builtin_amdgcn_ldexpf(1.f, -e);
#pragma unroll
            for (int j = 0; j < NKC; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    qf[j][x] = pack_f16_hw(__uint_as_float(qf[j][x] << 16) * f, __uint_as_float(qf[j][x] & 0xFFFF0000u) * f);
        }
#pragma unroll
        for (int j = 0; j < NKC; ++j) qf[j] = (qf[j] ^ qs.sign) & keep;
    }
    f32x16 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x16{};
    float m_ref = M0, l_run = 0.f;
    constexpr int PF = KV8 ? ACT_F16 : ACT_BF16;
    const char* const kl = lds.ring + kp * SB + (l32 >> 3) * 1024 + (l32 & 7) * 16 + (h32 ^ ((l32 >> 3) & 1)) * 128;
    const char* const vl = lds.ring + kp * SB + NKC * 1024 + (l32 >> 4) * 1024 + h32 * 256 + (l32 & 15) * 16;
    f32x16 sc;
    u32x4 p[2] = {u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}};
    auto key = [&](int at, int x) { return *(const u32x4*)(kl + at + (x >> 2) * 4096 + (x & 3) * 256); };
    auto value = [&](int at, int x) { return *(const u32x4*)(vl + at + x % NDT * 2048 + x / NDT * 512); };
    auto values = [&](int at) {                                // O += V P of the block in the slot at `at`
#pragma unroll
        for (int x = 0; x < NKC; ++x) o[x % NDT] = mfma32<PF>(value(at, x), p[x / NDT], o[x % NDT]);
    };
    // Both in turn, so that S, a chain, does not wait for itself; FD fragments are read ahead.
    auto both = [&](int before, int at) {
        constexpr int FD = 4;
        u32x4 f[FD];
        auto read = [&](int x) { f[x % FD] = x & 1 ? key(at, x >> 1) : value(before, x >> 1); };
#pragma unroll
        for (int x = 0; x < FD; ++x) read(x);
        sc = f32x16{};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2 * NKC; ++x) {
            const int y = x >> 1;
            if (x & 1) sc = mfma32<PF>(f[x % FD], qf[y], sc);
            else o[y % NDT] = mfma32<PF>(f[x % FD], p[y / NDT], o[y % NDT]);
            if (x + FD < 2 * NKC) read(x + FD);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto softmax = [&](int i) {
        const int past = (beg + i) * VT_BLK - sq.ctx;
        if (past > -VT_BLK || i >= n) {
            const uint32_t sees = i < n ? tree_sees(line, past) >> (4 * rare(h32)) : 0u;
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = sees >> (8 * (e >> 2) + (e & 3)) & 1 ? sc[e] : -INFINITY;
        }
        float t[5];
#pragma unroll
        for (int x = 0; x < 5; ++x) t[x] = fmaxf(fmaxf(sc[3 * x], sc[3 * x + 1]), sc[3 * x + 2]);
        t[0] = fmaxf(fmaxf(fmaxf(t[0], t[1]), t[2]), fmaxf(fmaxf(t[3], t[4]), sc[15]));
        // the other half's keys belong to the same rows
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(t[0]), __float_as_uint(t[0]), false, false);
        const float mx = fmaf(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), sl2, -BELOW<KV8>);
        const float m = mx > m_ref + LAZY ? mx : m_ref;
        if (__ballot(m != m_ref) != 0) {
            const float f = __builtin_amdgcn_exp2f(m_ref - m);
            l_run *= f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[dt] *= f;
        }
        m_ref = m;
        float ps[2] = {0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int e = 2 * x;
            const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[e], sl2, -m)), p1 = __builtin_amdgcn_exp2f(fmaf(sc[e + 1], sl2, -m));
            ps[0] += p0;
            ps[1] += p1;
            p[(e >> 2) & 1][((e & 3) >> 1) + 2 * (e >> 3)] = KV8 ? pack_f16_hw(p0, p1) : pack_bf16_hw(p0, p1);
        }
        l_run += ps[0] + ps[1];
    };
    auto meet = []() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // Step s sits in slot s % 3, s + 1 is stored while s is multiplied: in a slot that was done with before the barrier.
    auto run = [&](auto late, auto keys) {
        constexpr bool LATE = decltype(late)::value;
        auto put = [&](char* slot, int s, const Raw& r) {
            if (s * KP + KP > edge) store(slot, s, r, keys, Yes{});
            else store(slot, s, r, keys, No{});
        };
        // the values before step 0: zeros, times zero probabilities
        for (int x = tid; x < KP * NKC * 64; x += 512) *(u32x4*)(lds.ring + 2 * ST + x / (NKC * 64) * SB + NKC * 1024 + x % (NKC * 64) * 16) = u32x4{0u, 0u, 0u, 0u};
        put(lds.ring, 0, r0);
        fetch(2, r0, keys);
        meet();
        int at = 0;                                            // of step s
        auto step = [&](int s, Raw& r) {
            const int before = at == 0 ? 2 * ST : at - ST, after = at == 2 * ST ? 0 : at + ST;
            if (!LATE) both(before, at);
            if (s + 1 < steps) put(lds.ring + after, s + 1, r);
            fetch(s + 3, r, keys);
            if (!LATE) softmax(s * KP + kp);
            if (LATE) {
                if (s > 0) softmax((s - 1) * KP + kp);
                both(before, at);
            }
            meet();
            at = after;
        };
        int s = 0;
        for (; s + 1 < steps; s += 2) {
            step(s, r1);
            step(s + 1, r0);
        }
        if (s < steps) step(s, r1);
        if (LATE) softmax((steps - 1) * KP + kp);
        values(at == 0 ? 2 * ST : at - ST);
    };
    if (n > 0) {
        if (w < 4) run(No{}, Yes{});
        else run(Yes{}, No{});
    }

    // O^T element (dt, e) of lane l: dim 32 dt + 8 (e / 4) + 4 h32 + e % 4 of row l % 32.  The two sums of a row are merged.
    l_run += __shfl_xor(l_run, 32, 64);
    __syncthreads();
    const int wr = kp * RT + 32 * rg + l32;
    if (h32 == 0) {
        lds.mw[wr] = m_ref;
        lds.lw[wr] = l_run;
    }
    if (lane == 0) lds.sw[w] = strays;
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4)
            *(f32x4*)&lds.ow[wr * RS + 32 * dt + 8 * e4 + 4 * h32] = f32x4{o[dt][4 * e4], o[dt][4 * e4 + 1], o[dt][4 * e4 + 2], o[dt][4 * e4 + 3]};
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) any |= lds.sw[x];
    // a row's factors once, by a thread: of its two sums, and the whole's reference and sum.  (1 / l comes last, strays or not: rows
    // that see none of them keep their bits.)
    if (tid < RT) {
        const float m0 = lds.mw[tid], m1 = lds.mw[RT + tid], m = fmaxf(m0, m1);
        const float e0 = __builtin_amdgcn_exp2f(m0 - m), e1 = __builtin_amdgcn_exp2f(m1 - m);
        const float l = lds.lw[tid] * e0 + lds.lw[RT + tid] * e1;
        lds.mw[tid] = e0;
        lds.mw[RT + tid] = e1;
        lds.lw[tid] = 1.f / l;
        if (un.pieces > 1 && tid < rows) *(f32x2*)(a.ws + ((int64_t)un.part * RT + tid) * wst(D) + D) = f32x2{m, l};
    }
    __syncthreads();
#pragma unroll 4
    for (int it = tid; it < rows * (D / 4); it += 512) {
        const int c = it / (D / 4), d0 = it % (D / 4) * 4;
        f32x4 x = *(const f32x4*)&lds.ow[c * RS + d0] * lds.mw[c] + *(const f32x4*)&lds.ow[(RT + c) * RS + d0] * lds.mw[RT + c];
        const int r = row0 + c;
        if (any) {
#pragma unroll 1
            for (int e = 0; e < 4; ++e) {
                const float y = stray_sum<D, KV8, true>(a, b, kvh, d0 + e, max(beg, sq.ctx / VT_BLK) * VT_BLK,
                                                        min(sq.ctx + r / G, un.end * VT_BLK - 1), sq.ctx, lds.line[r / G]);
                x += f32x4{e == 0 ? y : 0.f, e == 1 ? y : 0.f, e == 2 ? y : 0.f, e == 3 ? y : 0.f};
            }
        }
        if (un.pieces == 1) {
            store4(a.out + ((int64_t)(sq.row0 + r / G) * a.n_heads + kvh * G + r % G) * D + d0, x * lds.lw[c], a.out_fmt);
        } else {
            *(f32x4*)(a.ws + ((int64_t)un.part * RT + c) * wst(D) + d0) = x;
        }
    }
}

}  // namespace

hipError_t launch_attn_wide(const AttnChunkArgs& a, unsigned grid, hipStream_t st) {
    if (a.kv.head_dim != D) return hipErrorInvalidValue;
    if (a.kv.format == FP_KV_INT8) FP_LAUNCH(attn_wide_kernel<true>, dim3(grid), dim3(512), 0, st, a);
    else FP_LAUNCH(attn_wide_kernel<false>, dim3(grid), dim3(512), 0, st, a);
    return hipGetLastError();
}

}  // namespace fpk
