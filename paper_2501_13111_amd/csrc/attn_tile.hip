// Chunk attention where sequences bring many rows to a kv head (a prompt's chunk, or a batch with one in it):
// tiles of 256 rows.  Rows, pieces and their join are those of attn_chunk.hip, whose tile_rows says when.
//
// A workgroup's four waves hold 64 rows each (two MFMA columns of 32) and walk the same 32-key blocks:
//     S^T = K Q^T,   O^T += V^T P^T,   l += 1 P^T        on MFMA 32x32x16
// The blocks pass through LDS as 16-bit fragments, each of which is read once per wave and feeds two
// products (64 rows per wave and not 32: LDS reads take matrix-core time, and the int8 unpacking is
// done once per 256 rows).  The sum l comes from the same rounded probabilities as O, on the matrix cores:
// where one key dominates, its rounding cancels.
//
// One wave per SIMD, so products and softmax overlap inside the wave: trip i multiplies S of block
// i + 1 and P V of block i - 1 while it takes the softmax of block i; none of them depends on another.
// A lone wave issues an instruction every five cycles or so and a product takes 32, so the trip is
// written out as a sequence of products, each followed by the five or so instructions that fit beside it,
// and its length is the number of its instructions.
//
// The softmax's reference m moves only when a score passes it by 2^LAZY, and then to 2^-BELOW of that
// score; the accumulators are rescaled then, outside the inner loop.  Probabilities are taken relative to m:
// at most 2^(LAZY + BELOW).  int8: 2^15, so that in fp16 those down to 2^-21 of the largest keep all their bits
// (smaller ones are off by 2^-32 of it at most).  bf16: 2^-ROOM (attn_stream.h), for values of any size.
//
// int8: keys and values are unpacked to fp16 with their scales (code * scale rounded to 11 bits, so that
// none may reach 65520: half the error that bf16's 8 bits leave in the output, and the matrix cores take no
// scale); queries are fp16 too, each row brought to the top of its range by a power of two that the scale takes
// back, so that only elements 2^-29 of the row's largest and smaller lose bits.
//
// 1024 tokens after 31744, 32 heads on 4 of 128, in a loop of 20 calls: bf16 523 us, 1.03 PFLOP/s of the 1.31 that a
// large library matrix product reaches; int8 633, 0.85 (its unpacking takes the instructions that the longer trip
// shows); heads of 64, bf16 360, 0.75 (half the products, the same softmax).  A trip of 36 products is 1152 cycles of matrix core and takes some
// 2000 (int8 2600).  A unit's fixed part is 6 us before the first trip (the plan 1.5, the rest the first blocks and
// queries at the memory's rate when every unit starts at once) and 2.5 after the last.
#include <type_traits>
#include <utility>

#include "attn_stream.h"
#include "lds_copy.h"

namespace fpk {

namespace {

constexpr float LAZY = 8.f;
template <bool KV8>
constexpr float BELOW = KV8 ? 7.f : -(LAZY + ROOM);
constexpr int RING = 8;                    // LDS slots
constexpr int AHEAD = 4;                   // blocks on their way (int8: in registers, two; unpacked two ahead)
constexpr int FD = 4;                      // fragments read ahead

// f(0), f(1), .. f(N - 1) with the index a constant.
template <class F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for(f, std::make_integer_sequence<int, N>{});
}

__device__ __forceinline__ uint32_t pk_mul(uint32_t x, uint32_t y) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) * __builtin_bit_cast(f16x2, y));
}
template <int D, bool KV8>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1))) attn_tile_kernel(AttnChunkArgs a) {
    constexpr int NKC = D / 16, NDT = D / 32, NVC = 2 * NDT, CH = NKC + NVC;
    constexpr int SB = CH * 1024;          // bytes of a slot: keys, then values
    constexpr int JPW = CH / 4;            // copies per block and wave (bf16)
    __shared__ __attribute__((aligned(1024))) char smem[RING * SB];

    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h32 = lane >> 5;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<TILE_ROWS, false, true>(a, G, un)) return;
    if (few_rows(un.sq, G)) {
        stream_unit<D, KV8, 1, true>(a, un, *(StreamLds<D, 1>*)smem);
        return;
    }
    const Seq& sq = un.sq;
    const int b = un.b, kvh = un.kvh, row0 = un.rt * TILE_ROWS, rows = min(TILE_ROWS, sq.n * G - row0);
    auto uni = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int beg = uni(un.beg), n = uni(max(un.end - un.beg, 0));
    // blocks that this wave's rows see, and that all of them see whole
    const int wr0 = row0 + 64 * w, wrows = min(max(rows - 64 * w, 0), 64);
    const int nw = uni(wrows > 0 ? min(n, (sq.ctx + (wr0 + wrows - 1) / G) / VT_BLK + 1 - beg) : 0);
    const int wfull = uni((sq.ctx + wr0 / G + 1) / VT_BLK - beg);
    // From block `edge` on some row of the tile does not see every key.  Values there that are not finite
    // would make NaN of its zero probabilities: they are taken out, and what they are to the rows that
    // do see them is written at the end.
    const int edge = uni((sq.ctx + row0 / G + 1) / VT_BLK - beg);
    __shared__ int sw[4];
    bool strays = false;                   // this wave has taken some out

    // ---- staging.  The pool blocks of 64 blocks at a time are held across the lanes.
    constexpr int KB = VT_BLK * D * (KV8 ? 1 : 2);
    int pbs = 0;
    auto pages = [&](int i0) {
        const int i = i0 + lane;
        pbs = i < n ? pool_block(a.kv, a.chunk, b, kvh, beg + i) : -1;
    };
    auto turn_pages = [&](int i) {
        if ((i & 63) == 0) pages(i);
    };
    auto block_of = [&](int i) { return __builtin_amdgcn_readlane(pbs, min(i, n - 1) & 63); };

    // LDS layout of a slot: keys in groups of 8 by 128 bytes of dims, chunk c of 16 bytes of key k at
    // 1024 (4 (c / 8) + k / 8) + 128 (c % 8, the low bit flipped in every other group) + 16 (k % 8);
    // values 16 dims a group, chunk c (8 slots) of dim d at 1024 (d / 16) + 256 c + 16 (d % 16).  A group is
    // one copy's kilobyte and whole cache lines of the pool, and the 16 lanes that read a fragment
    // together find their 16-byte pieces in 256 different bytes.
    //
    // bf16: copies straight into LDS, lower two waves keys, upper two values; past the last block the last
    // again, so that every trip issues the same number.
    static_assert(NKC == 2 * JPW && NVC == 2 * JPW, "two waves a kind");
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lvoid_t*)smem;
    const bool isv = w >= 2;
    const char* pool = isv ? (const char*)a.kv.v : (const char*)a.kv.k;
    const uint32_t v0 = isv ? (lane & 15) * (2 * VT_BLK) + (lane >> 4) * 16 : (lane & 7) * (2 * D) + (lane >> 3) * 16;
    const uint32_t voff[2] = {v0, isv ? v0 : v0 ^ 16u};
    i32x4 crs;                             // the copies' block and slot, for its JPW copies
    uint32_t cdst = 0;
    auto copy_begin = [&](int i) {
        const int pb = block_of(i);
        crs = rsrc_words(pool + (int64_t)max(pb, 0) * KB, pb >= 0 ? KB : 0);
        cdst = lds0 + (uint32_t)(i & (RING - 1)) * SB + (uint32_t)(w * JPW) * 1024u;
    };
    auto copy = [&](int x) {
        const uint32_t t = (isv ? w - 2 : w) * JPW + x;
        lds_copy<16>(crs, voff[x & 1], isv ? t * 1024u : (t & 3) * (16 * D) + (t >> 2) * 128u,
                     __builtin_amdgcn_readfirstlane(cdst + x * 1024));
    };
    // int8 (D = 128): a thread's 16 codes of a key and 16 slots of a value dim, and
    // their scales: one for the key, those of 16 positions for the values.
    struct Raw {
        u32x4 k, v, sa, sb;
        uint32_t ks;
    };
    static_assert(!KV8 || D == 128, "256 threads' pieces make a block");
    auto fetch = [&](int i, Raw& x) {
        const int pb = block_of(i);
        const int64_t at = max(pb, 0);
        const int ok = pb >= 0 ? 1 : 0;                    // a missing page reads as zeros
        const auto rk = buf_rsrc((const char*)a.kv.k + at * KB, ok * KB);
        const auto rv = buf_rsrc((const char*)a.kv.v + at * KB, ok * KB);
        const auto sk = buf_rsrc(a.kv.k_scales + at * VT_BLK, ok * 2 * VT_BLK);
        const auto sv = buf_rsrc(a.kv.v_scales + at * VT_BLK, ok * 2 * VT_BLK);
        const uint32_t j2 = tid / D & 1;
        x.k = __builtin_amdgcn_raw_buffer_load_b128(rk, (tid & 31) * D + 16 * (tid >> 5 & (D / 16 - 1)), 0, 0);
        x.v = __builtin_amdgcn_raw_buffer_load_b128(rv, (tid & (D - 1)) * VT_BLK + 16 * j2, 0, 0);
        x.ks = __builtin_amdgcn_raw_buffer_load_b16(sk, (tid & 31) * 2, 0, 0);
        x.sa = __builtin_amdgcn_raw_buffer_load_b128(sv, 16 * j2, 0, 0);          // keys 8 j2 .. + 7
        x.sb = __builtin_amdgcn_raw_buffer_load_b128(sv, 32 + 16 * j2, 0, 0);     // keys 16 + 8 j2 .. + 7
    };
    const int sa8 = (tid & 31) >> 3, sseg = tid >> 5 & (D / 16 - 1);
    char* const kst = smem + (4 * (sseg >> 2) + sa8) * 1024 + (2 * sseg & 7) * 128 + (tid & 7) * 16;
    char* const vst = smem + NKC * 1024 + ((tid & (D - 1)) >> 4) * 1024 + (tid / D & 1) * 512 + (tid & 15) * 16;
    // word x of a thread's keys (values): four codes unpacked; the two words of a piece make 16 bytes
    u32x2 half;
    auto stage_k = [&](int i, const Raw& r, int x) {
        const uint32_t s2 = r.ks | (r.ks << 16);
        const u32x2 c = i8x4_to_f16x4(r.k[x]);
        const u32x2 v = u32x2{pk_mul(c.x, s2), pk_mul(c.y, s2)};
        if ((x & 1) == 0) half = v;
        else
            *(u32x4*)(kst + (i & (RING - 1)) * SB + ((x >> 1) ^ (sa8 & 1)) * 128) = u32x4{half.x, half.y, v.x, v.y};
    };
    auto stage_v = [&](int i, const Raw& r, int x) {
        // slots 4 x .. 4 x + 3 of the 16: keys 4 (x / 2) + 16 (x % 2) + .. of the eight and eight that sa, sb hold
        const uint32_t s0 = (x & 1) ? r.sb[x & 2] : r.sa[x & 2], s1 = (x & 1) ? r.sb[(x & 2) + 1] : r.sa[(x & 2) + 1];
        const u32x2 c = i8x4_to_f16x4(r.v[x]);
        const u32x2 v = u32x2{pk_mul(c.x, s0), pk_mul(c.y, s1)};
        if ((x & 1) == 0) half = v;
        else *(u32x4*)(vst + (i & (RING - 1)) * SB + (x >> 1) * 256) = u32x4{half.x, half.y, v.x, v.y};
    };
    // Scales of positions past the sequence may be anything: zero in the block where it ends.
    // int8: values are finite if their scales are.
    auto clear_tail = [&](int i, Raw& r) {
        if constexpr (KV8) {
            if ((beg + i + 1) * VT_BLK > sq.len) {
                const int nk = sq.len - (beg + i) * VT_BLK - 8 * (tid / D & 1);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    r.sa[x] &= (2 * x < nk ? 0xFFFFu : 0u) | (2 * x + 1 < nk ? 0xFFFF0000u : 0u);
                    r.sb[x] &= (2 * x + 16 < nk ? 0xFFFFu : 0u) | (2 * x + 17 < nk ? 0xFFFF0000u : 0u);
                }
            }
            if (i >= edge) {
                uint32_t bad = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    bad |= nonfinite<F16_EXP>(r.sa[x]) | nonfinite<F16_EXP>(r.sb[x]);
                    r.sa[x] = finite_halves<F16_EXP>(r.sa[x]);
                    r.sb[x] = finite_halves<F16_EXP>(r.sb[x]);
                }
                strays |= __ballot(bad != 0) != 0;
            }
        }
    };
    auto stage = [&](int i, Raw& r) {
        clear_tail(i, r);
#pragma unroll
        for (int x = 0; x < 4; ++x) stage_k(i, r, x);
#pragma unroll
        for (int x = 0; x < 4; ++x) stage_v(i, r, x);
    };

    // bf16: a block's values in LDS, each wave a quarter, before the barrier that ends the trip.  Those of positions
    // past the sequence, which may be anything, become zeros first.
    auto scrub = [&](int i) {
        if constexpr (!KV8) {
            char* const v = smem + (i & (RING - 1)) * SB + NKC * 1024 + 16 * tid;
            const int nk = uni(sq.len - (beg + i) * VT_BLK);
            if (nk < VT_BLK) {
                const u32x4 keep = {slots_below((tid >> 4) & 3, 0, nk), slots_below((tid >> 4) & 3, 1, nk),
                                    slots_below((tid >> 4) & 3, 2, nk), slots_below((tid >> 4) & 3, 3, nk)};
#pragma unroll
                for (int x = 0; x < NVC / 4; ++x) *(u32x4*)(v + 4096 * x) &= keep;
            }
            uint32_t bad = 0;
#pragma unroll
            for (int x = 0; x < NVC / 4; ++x) {
                u32x4 y = *(const u32x4*)(v + 4096 * x);
                const uint32_t odd = nonfinite<BF16_EXP>(y.x) | nonfinite<BF16_EXP>(y.y) | nonfinite<BF16_EXP>(y.z) | nonfinite<BF16_EXP>(y.w);
                if (odd) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = finite_halves<BF16_EXP>(y[e]);
                    *(u32x4*)(v + 4096 * x) = y;
                }
                bad |= odd;
            }
            strays |= __ballot(bad != 0) != 0;
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    };
    // what trip i begins with: the next pages, and block i + 1, which the last barrier has made whole
    auto begin = [&](int i) {
        turn_pages(i + 4);
        if (!KV8 && i + 1 >= edge) scrub(i + 1);
    };

    // the first blocks are on their way while the queries are
    Raw ra, rb, r0, r1;
    if (n > 0) {
        pages(0);
        if constexpr (KV8) {
            fetch(0, r0);
            fetch(1, r1);
            fetch(2, ra);
            fetch(3, rb);
        } else {
            for (int i = 0; i < AHEAD; ++i) {
                copy_begin(i);
#pragma unroll
                for (int x = 0; x < JPW; ++x) copy(x);
            }
        }
    }

    // ---- queries: columns 32 c + l % 32 of the wave; a negative scale turns their signs
    u32x4 qf[2][NKC];
    int lim[2];                            // last position that the lane's row sees
    float sl2[2];                          // scores to base 2
    const QScale qs = q_scale(a.scale);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int rho = wr0 + 32 * c + l32;
        const bool live = 32 * c + l32 < wrows;
        const int tok = live ? rho / G : 0, h = live ? rho % G : 0;
        lim[c] = live ? sq.ctx + tok : -1;
        sl2[c] = qs.sl2;
        const uint16_t* q = a.q + (int64_t)(sq.row0 + tok) * a.q_stride + (kvh * G + h) * D;
        const uint32_t keep = live ? qs.keep : 0u, sign = qs.sign;
#pragma unroll
        for (int j = 0; j < NKC; ++j) qf[c][j] = *(const u32x4*)(q + 16 * j + 8 * h32);
        if constexpr (KV8) {
            float m = 0.f;
#pragma unroll
            for (int j = 0; j < NKC; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    m = fmaxf(m, fmaxf(fabsf(__uint_as_float(qf[c][j][x] << 16)), fabsf(__uint_as_float(qf[c][j][x] & 0xFFFF0000u))));
            m = fmaxf(m, __shfl_xor(m, 32, 64));
            // the row's largest to 2^14 .. 2^15 (2^-e stays finite: bf16's least, 2^-133, comes to 2^-7, exact); the
            // scale takes 2^e and stays a number above zero, which turns a masked score's -infinity into no NaN
            const int e = live && m > 0.f ? max(__builtin_amdgcn_frexp_expf(m) - 15, -126) : 0;
            sl2[c] = fminf(fmaxf(__builtin_amdgcn_ldexpf(sl2[c], e), 1.2e-38f), 3.4e38f);
            const float f = __builtin_amdgcn_ldexpf(1.f, -e);
#pragma unroll
            for (int j = 0; j < NKC; ++j)
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    qf[c][j][x] = pack_f16_hw(__uint_as_float(qf[c][j][x] << 16) * f, __uint_as_float(qf[c][j][x] & 0xFFFF0000u) * f);
        }
#pragma unroll
        for (int j = 0; j < NKC; ++j) {
            qf[c][j] = (qf[c][j] ^ sign) & keep;
            asm volatile("" : "+v"(qf[c][j]));   // loaded here, not inside the block loop
        }
    }

    f32x16 oacc[2][NDT], lacc[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        lacc[c] = f32x16{};
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) oacc[c][dt] = f32x16{};
    }
    float m_ref[2] = {M0, M0}, f[2] = {1.f, 1.f};
    struct S2 {
        f32x16 s[2];
    };
    struct P2 {
        u32x4 p[2][2];
    };
    const u32x4 ones = KV8 ? u32x4{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u}
                           : u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
    const char* kl = smem + (l32 >> 3) * 1024 + (l32 & 7) * 16 + (h32 ^ ((l32 >> 3) & 1)) * 128;
    const char* vl = smem + NKC * 1024 + (l32 >> 4) * 1024 + h32 * 256 + (l32 & 15) * 16;
    auto kfrag = [&](int sl, int j) { return *(const u32x4*)(kl + sl * SB + (j >> 2) * 4096 + (j & 3) * 256); };
    auto vfrag = [&](int sl, int x) { return *(const u32x4*)(vl + sl * SB + (x % NDT) * 2048 + (x / NDT) * 512); };
    // A trip's fragments in order: the values of block i - 1, then the keys of block i + 1; read FD
    // ahead, across trips too.
    u32x4 fr[8];
    auto read = [&](int x, int i) {
        const int sl = (x < NVC ? i - 1 : i + 1) & (RING - 1);
        fr[x & 7] = x < NVC ? vfrag(sl, x) : kfrag(sl, x - NVC);
    };
    // S goes to vector registers, where the softmax reads it (the compiler would accumulate it, like O,
    // in accumulation registers and copy it over in every trip).  It does not see this product's latency:
    // settle() lies between the last one of a trip and the next trip's first use.
    auto mfma_s = [](f32x16& d, const u32x4& k, const u32x4& q, bool zero) {
        if constexpr (KV8) {
            if (zero) asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, 0" : "=&v"(d) : "v"(k), "v"(q));
            else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(d) : "v"(k), "v"(q));
        } else {
            if (zero) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(d) : "v"(k), "v"(q));
            else asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(d) : "v"(k), "v"(q));
        }
    };
    constexpr int PF = KV8 ? ACT_F16 : ACT_BF16;
    auto settle = []() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); };
    auto koff = [](int e) { return 8 * (e >> 2) + (e & 3); };

    // ---- trip i: scores cur -> probabilities pout; scores of block i + 1 -> nxt; pin (block i - 1)
    // times its values.  A share's instructions are independent of each other (a lone wave waits for
    // a result that it uses at once): the maxima as trees, the references, then for pairs of elements the
    // exponent's argument, its power and its rounding, each one product later; between them the
    // staging of a later block.
    auto trip = [&](int i, S2& cur, S2& nxt, const P2& pin, P2& pout, Raw& raw, auto dm) {
        constexpr bool DM = decltype(dm)::value;
        constexpr int NS = CH + 2, NY = 2 * NS;                       // steps, products
        constexpr int YM = D == 128 ? 6 : 3;                          // products beside maxima and references
        float t[2][5], m[2];
        auto max3 = [](float x, float y, float z) { return fmaxf(fmaxf(x, y), z); };
        auto max_a = [&](int c) {
            if constexpr (DM) {
                const int lc = lim[c] - (beg + i) * VT_BLK - 4 * h32;
#pragma unroll
                for (int e = 0; e < 16; ++e) cur.s[c][e] = koff(e) <= lc ? cur.s[c][e] : -INFINITY;
            }
#pragma unroll
            for (int x = 0; x < 5; ++x) t[c][x] = max3(cur.s[c][3 * x], cur.s[c][3 * x + 1], cur.s[c][3 * x + 2]);
        };
        auto max_b = [&](int c) {
            t[c][0] = max3(t[c][0], t[c][1], t[c][2]);
            t[c][1] = max3(t[c][3], t[c][4], cur.s[c][15]);
        };
        auto max_c = [&](int c) { t[c][0] = fmaf(fmaxf(t[c][0], t[c][1]), sl2[c], -BELOW<KV8>); };
        auto ref_a = [&](int c) {          // the other half's keys belong to the same rows
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(t[c][0]), __float_as_uint(t[c][0]), false, false);
            t[c][0] = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
            t[c][1] = m_ref[c] + LAZY;
        };
        auto ref_b = [&](int c) {
            m[c] = t[c][0] > t[c][1] ? t[c][0] : m_ref[c];
            f[c] = m_ref[c] - m[c];
            m_ref[c] = m[c];
        };
        auto arg = [&](int x) {
            const int c = x >> 3, e = 2 * (x & 7);
            cur.s[c][e] = fmaf(cur.s[c][e], sl2[c], -m[c]);
            cur.s[c][e + 1] = fmaf(cur.s[c][e + 1], sl2[c], -m[c]);
        };
        auto power = [&](int x) {
            const int c = x >> 3, e = 2 * (x & 7);
            cur.s[c][e] = __builtin_amdgcn_exp2f(cur.s[c][e]);
            cur.s[c][e + 1] = __builtin_amdgcn_exp2f(cur.s[c][e + 1]);
        };
        auto round = [&](int x) {
            const int c = x >> 3, e = 2 * (x & 7);
            pout.p[c][(e >> 2) & 1][((e & 3) >> 1) + 2 * (e >> 3)] =
                KV8 ? pack_f16_hw(cur.s[c][e], cur.s[c][e + 1]) : pack_bf16_hw(cur.s[c][e], cur.s[c][e + 1]);
        };
        // what goes beside product y
        auto share = [&](auto y) {
            if constexpr (YM == 6) {
                if (y == 0) max_a(0);
                if (y == 1) max_a(1);
                if (y == 2) { max_b(0); max_b(1); }
                if (y == 3) { max_c(0); max_c(1); }
                if (y == 4) { ref_a(0); ref_a(1); }
                if (y == 5) { ref_b(0); ref_b(1); }
            } else {
                if (y == 0) { max_a(0); max_a(1); }
                if (y == 1) { max_b(0); max_b(1); max_c(0); max_c(1); }
                if (y == 2) { ref_a(0); ref_a(1); ref_b(0); ref_b(1); }
            }
            static_for<16>([&](auto x) {
                constexpr int at = YM + x * (NY - 2 - YM) / 16;
                if (y == at + 2) round(x);
                if (y == at + 1) power(x);
                if (y == at) arg(x);
            });
            if (y == YM + 3) {
                f[0] = __builtin_amdgcn_exp2f(f[0]);
                f[1] = __builtin_amdgcn_exp2f(f[1]);
            }
            if constexpr (KV8) {
                static_for<8>([&](auto x) {
                    if (y == YM + x * (NY - 2 - YM) / 8) {
                        if constexpr (x < 4) stage_k(i + 2, raw, x);
                        else stage_v(i + 2, raw, x - 4);
                    }
                });
                if (y == NY - 1) fetch(i + 4, raw);
            } else {
                if (y == 1) copy_begin(i + AHEAD);
                static_for<JPW>([&](auto x) {
                    if (y == YM + 2 + 3 * x) copy(x);
                });
            }
        };
        static_for<NY>([&](auto y) {
            constexpr int s = y / 2, c = y & 1;
            constexpr bool isV = s < NVC + 2, one = isV && s % (NDT + 1) == NDT;
            constexpr int j2 = isV ? s / (NDT + 1) : 0, dt = s % (NDT + 1);
            constexpr int x = isV ? j2 * NDT + (one ? 0 : dt) : s - 2;       // fragment
            if constexpr (c == 0 && !one) {
                if constexpr (x + FD < CH) read(x + FD, i);
                else read(x + FD - CH, i + 1);
            }
            if constexpr (one) lacc[c] = mfma32<PF>(ones, pin.p[c][j2], lacc[c]);
            else if constexpr (isV) oacc[c][dt] = mfma32<PF>(fr[x & 7], pin.p[c][j2], oacc[c][dt]);
            else mfma_s(nxt.s[c], fr[x & 7], qf[c][x - NVC], x == NVC);
            __builtin_amdgcn_sched_barrier(0);
            share(y);
            __builtin_amdgcn_sched_barrier(0);
        });
        share(std::integral_constant<int, NY>{});
        settle();
    };
    // Trips end with every wave's block i + 2 in LDS.
    auto meet = [&]() {
        if constexpr (KV8) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(2 * JPW) : "memory");
    };
    using T_ = std::integral_constant<bool, true>;
    using F_ = std::integral_constant<bool, false>;

    if (n > 0) {
        auto swap_raw = [&]() {
            auto swap = [](auto& x, auto& y) {
                const auto z = x;
                x = y;
                y = z;
            };
            if constexpr (KV8) {
                swap(ra.k, rb.k);
                swap(ra.v, rb.v);
                swap(ra.sa, rb.sa);
                swap(ra.sb, rb.sb);
                swap(ra.ks, rb.ks);
            }
        };
        // zeros before block 0: trip 0 multiplies them by zero probabilities
        for (int x = tid; x < NVC * 64; x += 256) *(u32x4*)(smem + (RING - 1) * SB + NKC * 1024 + 16 * x) = u32x4{0u, 0u, 0u, 0u};
        if constexpr (KV8) {
            stage(0, r0);
            stage(1, r1);
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        } else {
            // blocks 0 and 1
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * JPW) : "memory");
            if (edge <= 0) {
                scrub(0);
                asm volatile("s_barrier" ::: "memory");
            }
        }
        int i = 0;
        if (nw > 0) {
            S2 cur, nxt;
            P2 pa, pb;
#pragma unroll
            for (int j = 0; j < NKC; ++j) {
                const u32x4 k = kfrag(0, j);
                mfma_s(cur.s[0], k, qf[0][j], j == 0);
                mfma_s(cur.s[1], k, qf[1][j], j == 0);
            }
            settle();
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int j = 0; j < 2; ++j) pa.p[c][j] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int x = 0; x < FD; ++x) read(x, 0);
            auto grown = [&]() { return __ballot(f[0] != 1.f || f[1] != 1.f) != 0; };
            // after one trip instead of two: the registers that the next turn starts from
            auto turn = [&]() {
                cur = nxt;
                pa = pb;
                swap_raw();
            };
            // Two trips a turn, scores, probabilities and raw codes changing registers.  The loop is left for
            // a new reference: the accumulators are rescaled out here, so that in there only the products
            // touch them.
            const int ne = min(wfull, nw);
            while (i < nw) {
                bool more = false;
                while (!more && i + 1 < ne) {
                    begin(i);
                    clear_tail(i + 2, ra);
                    trip(i, cur, nxt, pa, pb, ra, F_{});
                    meet();
                    ++i;
                    more = grown();
                    if (!more) {
                        begin(i);
                        clear_tail(i + 2, rb);
                        trip(i, nxt, cur, pb, pa, rb, F_{});
                        meet();
                        ++i;
                        more = grown();
                    } else {
                        turn();
                    }
                }
                while (!more && i < nw) {
                    begin(i);
                    clear_tail(i + 2, ra);
                    trip(i, cur, nxt, pa, pb, ra, T_{});
                    meet();
                    ++i;
                    turn();
                    more = grown();
                }
                // in accumulation registers, four at a time (multiplied in plain code, all of them would move
                // to vector registers, and be copied in the loop)
                static_for<2>([&](auto c) {
                    static_for<NDT + 1>([&](auto dd) {
                        static_for<4>([&](auto ee) {
                            constexpr int e = 4 * ee, dt = dd;
                            f32x16& acc = dt < NDT ? oacc[c][dt < NDT ? dt : 0] : lacc[c];
                            float x0 = acc[e], x1 = acc[e + 1], x2 = acc[e + 2], x3 = acc[e + 3], v0, v1, v2, v3;
                            asm volatile("v_accvgpr_read_b32 %4, %0\n\tv_accvgpr_read_b32 %5, %1\n\t"
                                         "v_accvgpr_read_b32 %6, %2\n\tv_accvgpr_read_b32 %7, %3\n\t"
                                         "v_mul_f32 %4, %4, %8\n\tv_mul_f32 %5, %5, %8\n\tv_mul_f32 %6, %6, %8\n\tv_mul_f32 %7, %7, %8\n\t"
                                         "v_accvgpr_write_b32 %0, %4\n\tv_accvgpr_write_b32 %1, %5\n\t"
                                         "v_accvgpr_write_b32 %2, %6\n\tv_accvgpr_write_b32 %3, %7"
                                         : "+a"(x0), "+a"(x1), "+a"(x2), "+a"(x3), "=&v"(v0), "=&v"(v1), "=&v"(v2), "=&v"(v3)
                                         : "v"(f[c]));
                            acc[e] = x0;
                            acc[e + 1] = x1;
                            acc[e + 2] = x2;
                            acc[e + 3] = x3;
                        });
                    });
                });
                asm volatile("s_nop 4" ::: "memory");      // before a product adds to them
            }
            // the last block's values
#pragma unroll
            for (int x = 0; x < NVC; ++x) {
                const u32x4 v = vfrag((nw - 1) & (RING - 1), x);
                oacc[0][x % NDT] = mfma32<PF>(v, pa.p[0][x / NDT], oacc[0][x % NDT]);
                oacc[1][x % NDT] = mfma32<PF>(v, pa.p[1][x / NDT], oacc[1][x % NDT]);
            }
#pragma unroll
            for (int j2 = 0; j2 < 2; ++j2) {
                lacc[0] = mfma32<PF>(ones, pa.p[0][j2], lacc[0]);
                lacc[1] = mfma32<PF>(ones, pa.p[1][j2], lacc[1]);
            }
        }
        for (; i < n; ++i) {               // a wave past its rows keeps staging
            begin(i);
            if constexpr (KV8) {
                stage(i + 2, ra);
                fetch(i + 4, ra);
                swap_raw();
            } else {
                copy_begin(i + AHEAD);
#pragma unroll
                for (int x = 0; x < JPW; ++x) copy(x);
            }
            meet();
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // no copy outlives the workgroup
    }

    // O^T element (dt, e) of lane l: dim 32 dt + 8 (e / 4) + 4 h32 + e % 4 of row 32 c + l % 32
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float l = lacc[c][0];
        if (32 * c + l32 >= wrows) continue;
        const int rho = wr0 + 32 * c + l32;
        if (un.pieces == 1) {
            const float inv = 1.f / l;
            uint16_t* orow = a.out + ((int64_t)(sq.row0 + rho / G) * a.n_heads + kvh * G + rho % G) * D;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4)
                    store4(orow + 32 * dt + 8 * e4 + 4 * h32,
                           f32x4{oacc[c][dt][4 * e4], oacc[c][dt][4 * e4 + 1], oacc[c][dt][4 * e4 + 2], oacc[c][dt][4 * e4 + 3]} * inv, a.out_fmt);
        } else {
            // a piece: the accumulators as the lanes hold them (whole kilobytes), then (m, l) of each row
            float* dst = a.ws + (int64_t)un.part * TILE_ROWS * wst(D);
            f32x4* od = (f32x4*)(dst + tile_part<D>(64 * w + 32 * c + l32, 4 * h32));
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
                for (int e4 = 0; e4 < 4; ++e4)
                    od[(4 * dt + e4) * 64] =
                        f32x4{oacc[c][dt][4 * e4], oacc[c][dt][4 * e4 + 1], oacc[c][dt][4 * e4 + 2], oacc[c][dt][4 * e4 + 3]};
            if (h32 == 0) *(f32x2*)(dst + TILE_ROWS * D + 2 * (64 * w + 32 * c + l32)) = f32x2{m_ref[c], l};
        }
    }
    // what the values taken out are to the rows that see them
    if (edge < n) {
        if (lane == 0) sw[w] = strays;
        __syncthreads();
        if ((sw[0] | sw[1] | sw[2] | sw[3]) == 0) return;
        for (int x = 0; x < 2 * (D / 2); ++x) {
            const int c = x & 1, d = 8 * (x >> 3) + 4 * h32 + ((x >> 1) & 3), r = 32 * c + l32;
            if (r >= wrows) continue;
            const int seen = sq.ctx + (wr0 + r) / G;
            const float sum = stray_sum<D, KV8>(a, b, kvh, d, (beg + max(edge, 0)) * VT_BLK, min(seen, (beg + n) * VT_BLK - 1));
            if (sum == 0.f) continue;
            // added to what the lane wrote there, which may be infinite or NaN too
            if (un.pieces == 1) {
                uint16_t* p = a.out + ((int64_t)(sq.row0 + (wr0 + r) / G) * a.n_heads + kvh * G + (wr0 + r) % G) * D + d;
                *p = act_store(sum + act_load(*p, a.out_fmt), a.out_fmt);
            } else {
                a.ws[(int64_t)un.part * TILE_ROWS * wst(D) + tile_part<D>(64 * w + r, d & ~3) + (d & 3)] += sum;
            }
        }
    }
}

// Joins the pieces of split tiles: D / 4 workgroups a tile, a thread per four dims of a row in the order
// that the pieces are stored.
template <int D>
__global__ void __launch_bounds__(256) attn_tile_join_kernel(AttnChunkArgs a) {
    constexpr int NDT = D / 32;
    const int nkv = a.kv.n_kv_heads, G = a.n_heads / nkv;
    Unit un;
    if (!find_unit<TILE_ROWS, true, false>(a, G, un)) return;
    const int it = blockIdx.y * 256 + threadIdx.x, lane = it & 63;
    const int chunk = (it >> 6) % (4 * NDT), row = 32 * (it / (256 * NDT)) + (lane & 31);
    const int rows = min(TILE_ROWS, un.sq.n * G - un.rt * TILE_ROWS);
    if (row >= rows) return;
    const int tiles = (un.sq.n * G + TILE_ROWS - 1) / TILE_ROWS;
    const float* src = a.ws + (int64_t)un.part * TILE_ROWS * wst(D);
    const int64_t step = (int64_t)tiles * TILE_ROWS * wst(D);
    float m = M0, l = 0.f;
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < un.pieces; i0 += 4) {
        f32x2 ml[4];
        f32x4 oi[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float* p = src + min(i0 + j, un.pieces - 1) * step;
            ml[j] = *(const f32x2*)(p + TILE_ROWS * D + 2 * row);
            oi[j] = ((const f32x4*)p)[it];
            if (i0 + j >= un.pieces) {
                ml[j] = f32x2{M0, 0.f};
                oi[j] = f32x4{0.f, 0.f, 0.f, 0.f};     // not the last piece's infinite sums again
            }
        }
        float mn = m;
#pragma unroll
        for (int j = 0; j < 4; ++j) mn = fmaxf(mn, ml[j][0]);
        const float f = __builtin_amdgcn_exp2f(m - mn);
        l *= f;
        o *= f;
        m = mn;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float e = __builtin_amdgcn_exp2f(ml[j][0] - m);
            l += ml[j][1] * e;
            o += oi[j] * e;
        }
    }
    const int rho = un.rt * TILE_ROWS + row;
    store4(a.out + ((int64_t)(un.sq.row0 + rho / G) * a.n_heads + un.kvh * G + rho % G) * D + 32 * (chunk >> 2) + 8 * (chunk & 3) +
               4 * (lane >> 5), o * (1.f / l), a.out_fmt);
}

}  // namespace

hipError_t launch_attn_tile(const AttnChunkArgs& a, unsigned grid, unsigned split_tiles, hipStream_t st) {
    const bool i8 = a.kv.format == FP_KV_INT8;
    const int D = a.kv.head_dim;
    if (D == 64 && i8) return hipErrorInvalidValue;
    if (D == 64) FP_LAUNCH((attn_tile_kernel<64, false>), dim3(grid), dim3(256), 0, st, a);
    else if (i8) FP_LAUNCH((attn_tile_kernel<128, true>), dim3(grid), dim3(256), 0, st, a);
    else FP_LAUNCH((attn_tile_kernel<128, false>), dim3(grid), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || split_tiles == 0) return e;
    if (D == 128) FP_LAUNCH(attn_tile_join_kernel<128>, dim3(split_tiles, D / 4), dim3(256), 0, st, a);
    else FP_LAUNCH(attn_tile_join_kernel<64>, dim3(split_tiles, D / 4), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace fpk
