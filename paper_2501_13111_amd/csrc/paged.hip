// Writing a chunk's keys and values into a paged cache (with the rotary embedding and the int8
// quantisation of the handle's own cache), and reading positions back.
//
// Both kernels take one workgroup per (32-position block touched, kv head): a block of values is
// transposed in the cache ([d][32 slots]), so it passes through LDS and moves in 16-byte pieces on
// both sides.  A thread holds eight dims of a position's lower half and the eight they are rotated
// with; the 8 (d = 64: 4) threads of a position find its largest magnitude by shuffles.  In an
// append the workgroup also rotates the queries of its kv head's group for the block's positions,
// whose cosines and sines it has just read.  Bound by memory: a long chunk's rows move once in, once
// out.  Appending 16 chunks of up to 4096, 32 heads on 8 of 128, bf16 (40,604 rows, 1.02 GB): 214 us, 4.8 TB/s; 64 single tokens on
// 8 heads, int8: 6.2 us, a chain of latencies.  Reading 8 sequences of up to 16000 back, 8 heads of 128, int8 (473 MB): 97 us, 4.9 TB/s.
#include "tree.h"

namespace fpk {

namespace {

constexpr int T = 256;

// 32-position blocks that the sequence's rows touch
__device__ __forceinline__ int seq_blocks(const Seq& s) {
    return s.n > 0 ? (s.len - 1) / VT_BLK - s.ctx / VT_BLK + 1 : 0;
}

// Room for the blocks of b sequences with r rows together: a sequence's n rows touch at most n / 32 + 2 blocks, and never more
// than n.  Sequence b's begin at that of its first row, so a workgroup finds them by row_start alone.
__host__ __device__ __forceinline__ int64_t blocks_before(int r, int b) {
    const int64_t few = (int64_t)r / VT_BLK + 2 * (int64_t)b;
    return few < r ? few : r;
}
// The sequence of block u, with u counted from its first block then; -1 if u is none.
__device__ __forceinline__ int find_block(const fp_chunk& c, int& u, Seq& sq) {
    auto before = [&](int b) { return (int)blocks_before(min(max(c.row_start[b], 0), c.n_rows), b); };
    const int b = last_at_most(c.n_seqs, u, before);
    if (b < 0) return -1;
    u -= before(b);
    sq = load_seq(c, b);
    return u >= 0 && u < seq_blocks(sq) ? b : -1;      // below 0: starts that decrease
}

// The workgroup's block and kv head.  Workgroup i runs on XCD i % 8: the heads of a block follow each other on one,
// whose L2 fetches the block's angles once.
__device__ __forceinline__ void unit(int nkv, int& u, int& kvh) {
    const int k = blockIdx.x >> 3;
    u = k / nkv * 8 + (blockIdx.x & 7);
    kvh = k % nkv;
}

__device__ __forceinline__ void unpack8(u32x4 v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
    return u32x4{pack_bf16_hw(x[0], x[1]), pack_bf16_hw(x[2], x[3]), pack_bf16_hw(x[4], x[5]), pack_bf16_hw(x[6], x[7])};
}

// Eight values at p: bf16, or the sum of ks fp32 partials pstride apart, in increasing order.
template <bool F32>
__device__ __forceinline__ void load8(const void* base, int64_t off, int ks, int64_t pstride, float (&x)[8]) {
    if constexpr (F32) {
        const float* p = (const float*)base + off;
        f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll 4
        for (int s = 1; s < ks; ++s) {
            a += *(const f32x4*)(p + s * pstride);
            b += *(const f32x4*)(p + s * pstride + 4);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    } else {
        unpack8(*(const u32x4*)((const uint16_t*)base + off), x);
    }
}

// x / s rounded.  Under a scale that is zero, infinite or NaN codes are zero: the last two read back as NaN.
__device__ __forceinline__ int8_t code8(float x, float s) {
    return s > 0.f && s < INFINITY ? (int8_t)(int)fminf(fmaxf(rintf(__fdiv_rn(x, s)), -127.f), 127.f) : (int8_t)0;
}
__device__ __forceinline__ u32x2 codes8(const float (&x)[8], float s) {
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)(uint8_t)code8(x[i], s) << (8 * (i & 3));
    return u32x2{w[0], w[1]};
}

// rotate_pair rounds one product and fuses the other with the sum, whatever the compiler contracts
__device__ __forceinline__ void rotate8(float (&lo)[8], float (&hi)[8], const float* c, const float* s) {
    const f32x4 c0 = *(const f32x4*)c, c1 = *(const f32x4*)(c + 4), s0 = *(const f32x4*)s, s1 = *(const f32x4*)(s + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float cc = i < 4 ? c0[i & 3] : c1[i & 3], ss = i < 4 ? s0[i & 3] : s1[i & 3];
        float l, h;
        rotate_pair(lo[i], hi[i], cc, ss, l, h);
        lo[i] = l;
        hi[i] = h;
    }
}

// int8 from bf16 inputs: the registers fit eight waves a SIMD only if the compiler is told (256 single tokens on 8 heads of
// 64 7.8 us, with seven waves 8.8).  bf16 caches have eight without it (16 chunks of up to 4096 214 us, told so 221).
// TREE: the rows are nodes of trees, rotated by the context's length and their depth.
template <int D, bool KV8, bool F32, bool TREE>
__global__ void __launch_bounds__(T, KV8 && !F32 ? 8 : 1) kv_append_paged_kernel(KvAppendArgs a) {
    constexpr int HALF = D / 2, NP = HALF / 8;             // threads per position
    constexpr int ES = KV8 ? 1 : 2;
    constexpr int VS = VT_BLK * ES + 16;                   // LDS bytes per value dim
    __shared__ __attribute__((aligned(16))) char vt[D * VS];
    const int tid = threadIdx.x;
    int u, kvh;
    unit(a.kv.n_kv_heads, u, kvh);
    Seq sq;
    const int b = find_block(a.chunk, u, sq);
    if (b < 0) return;
    const int blk = sq.ctx / VT_BLK + u;
    const int t0 = max(sq.ctx - blk * VT_BLK, 0), t1 = min(sq.len - blk * VT_BLK, VT_BLK);   // live positions
    const int np = t1 - t0;
    const int pb = pool_block(a.kv, a.chunk, b, kvh, blk);
    const int row0 = sq.row0 + (blk * VT_BLK + t0 - sq.ctx);
    const int G = a.q != nullptr ? a.n_heads / a.kv.n_kv_heads : 0;
    __shared__ int turn[TREE ? VT_BLK : 1];                // the live positions' rotary positions
    if constexpr (TREE) {
        if (tid < 64) {
            const int depth = __popcll(tree_lines(a.parent, sq)) - 1, i = tid - (row0 - sq.row0);
            if (tid < sq.n && i >= 0 && i < np) turn[i] = sq.ctx + depth;
        }
        __syncthreads();
    }

    for (int it = tid; it < (2 + G) * np * NP; it += T) {
        const int what = it / (np * NP), r = it % (np * NP);
        const int i = r / NP, j = 8 * (r % NP);
        const int t = t0 + i;
        const int64_t row = row0 + i;
        const int h = what < 2 ? kvh : kvh * G + what - 2;
        const void* src = what == 0 ? a.k : what == 1 ? a.v : a.q;
        const int64_t off = row * (what < 2 ? a.kv_stride : a.q_stride) + (int64_t)h * D + j;
        float lo[8], hi[8];
        load8<F32>(src, off, a.ks, a.pstride, lo);
        load8<F32>(src, off + HALF, a.ks, a.pstride, hi);
        if (what != 1 && a.cos_t != nullptr) {
            const int pos = TREE ? turn[i] : blk * VT_BLK + t;
            rotate8(lo, hi, a.cos_t + (int64_t)pos * HALF + j, a.sin_t + (int64_t)pos * HALF + j);
        }
        if (what >= 2) {
            uint16_t* q = a.q_out + (row * a.n_heads + h) * D + j;
            *(u32x4*)q = pack8(lo);
            *(u32x4*)(q + HALF) = pack8(hi);
            continue;
        }
        float sc = 0.f;
        if constexpr (KV8) {
            float m = 0.f;                                 // NaN if one of them is (fmaxf would drop it)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = __builtin_elementwise_maximum(m, __builtin_elementwise_maximum(fabsf(lo[e]), fabsf(hi[e])));
#pragma unroll
            for (int o = 1; o < NP; o <<= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, o, NP));
            const uint16_t sh = f2h(__fdiv_rn(m, 127.0f));
            sc = h2f(sh);
            if (j == 0 && pb >= 0) (what == 0 ? a.kv.k_scales : a.kv.v_scales)[(int64_t)pb * VT_BLK + t] = sh;
        }
        if (what == 0) {
            if (pb < 0) continue;
            char* dst = (char*)a.kv.k + ((int64_t)pb * VT_BLK + t) * D * ES;
            if constexpr (KV8) {
                *(u32x2*)(dst + j) = codes8(lo, sc);
                *(u32x2*)(dst + j + HALF) = codes8(hi, sc);
            } else {
                *(u32x4*)(dst + 2 * j) = pack8(lo);
                *(u32x4*)(dst + 2 * (j + HALF)) = pack8(hi);
            }
        } else {
            const int slot = vt_slot(t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if constexpr (KV8) {
                    *(int8_t*)(vt + (j + e) * VS + slot) = code8(lo[e], sc);
                    *(int8_t*)(vt + (j + e + HALF) * VS + slot) = code8(hi[e], sc);
                } else {
                    *(__bf16*)(vt + (j + e) * VS + 2 * slot) = (__bf16)lo[e];
                    *(__bf16*)(vt + (j + e + HALF) * VS + 2 * slot) = (__bf16)hi[e];
                }
            }
        }
    }
    __syncthreads();
    if (pb < 0) return;
    // values: 16-byte pieces of 16 / ES slots where every position is the chunk's, else element by
    // element (the block's other positions are earlier tokens')
    char* dst = (char*)a.kv.v + (int64_t)pb * D * VT_BLK * ES;
    if (np == VT_BLK) {
        constexpr int PD = VT_BLK * ES / 16;               // pieces per dim
        for (int it = tid; it < D * PD; it += T)
            *(u32x4*)(dst + 16 * it) = *(const u32x4*)(vt + it / PD * VS + it % PD * 16);
    } else {
        // a thread's position stays the same: those of a dim take the next power of two of neighbouring threads (40 sequences' up to 27 rows,
        // 8 heads of 128, int8, four layers and their move and read back: 52.8 us with a division for each element, 50.7)
        int th = tid;
        asm volatile("" : "+v"(th));                       // (computed above the loops this would cost them registers)
        const int lg = np > 1 ? 32 - __builtin_clz(np - 1) : 0, i = th & ((1 << lg) - 1), slot = vt_slot(t0 + i);
        if (i < np) {
            for (int dim = th >> lg; dim < D; dim += T >> lg) {
                if constexpr (KV8) dst[dim * VT_BLK + slot] = vt[dim * VS + slot];
                else *(uint16_t*)(dst + 2 * (dim * VT_BLK + slot)) = *(const uint16_t*)(vt + dim * VS + 2 * slot);
            }
        }
    }
}

template <int D, bool KV8>
__global__ void __launch_bounds__(T) kv_read_paged_kernel(KvReadArgs a) {
    constexpr int NP = D / 8, ES = KV8 ? 1 : 2, PD = VT_BLK * ES / 16;
    constexpr int VS = VT_BLK * ES + 16;
    __shared__ __attribute__((aligned(16))) char vt[D * VS];
    const int tid = threadIdx.x;
    int u, kvh;
    unit(a.kv.n_kv_heads, u, kvh);
    Seq sq;
    const int b = find_block(a.chunk, u, sq);
    if (b < 0) return;
    const int blk = sq.ctx / VT_BLK + u;
    const int t0 = max(sq.ctx - blk * VT_BLK, 0), t1 = min(sq.len - blk * VT_BLK, VT_BLK);
    const int np = t1 - t0;
    const int pb = pool_block(a.kv, a.chunk, b, kvh, blk);
    const int64_t row0 = sq.row0 + (blk * VT_BLK + t0 - sq.ctx);
    const int64_t prow = (int64_t)pb * VT_BLK;
    if (pb >= 0) {
        const u32x4* src = (const u32x4*)((const char*)a.kv.v + (int64_t)pb * D * VT_BLK * ES);
        for (int it = tid; it < D * PD; it += T) *(u32x4*)(vt + it / PD * VS + it % PD * 16) = src[it];
    }
    __syncthreads();
    auto store = [&](uint16_t* out, int i, int j, const float (&x)[8]) {
        *(u32x4*)(out + ((row0 + i) * a.kv.n_kv_heads + kvh) * D + j) = pack8(x);
    };
    if (tid < T / 2) {
        // values: four positions, whose slots are neighbours, of eight dims at a time
        for (int it = tid; it < VT_BLK / 4 * NP; it += T / 2) {
            const int t = it / NP * 4, j = 8 * (it % NP);
            if (t + 4 <= t0 || t >= t1) continue;
            constexpr int W = ES;                          // words of four values
            uint32_t c[8][W];
#pragma unroll
            for (int e = 0; e < 8; ++e)
#pragma unroll
                for (int w = 0; w < W; ++w) c[e][w] = pb >= 0 ? *(const uint32_t*)(vt + (j + e) * VS + ES * vt_slot(t) + 4 * w) : 0u;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                if (t + p < t0 || t + p >= t1) continue;
                float x[8];
                const float s = KV8 && pb >= 0 ? h2f(a.kv.v_scales[prow + t + p]) : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (KV8) x[e] = (float)(int8_t)(c[e][0] >> (8 * p)) * s;
                    else x[e] = __uint_as_float(p & 1 ? c[e][p >> 1] & 0xFFFF0000u : c[e][p >> 1] << 16);
                }
                store(a.v_out, t + p - t0, j, x);
            }
        }
    } else {
        for (int it = tid - T / 2; it < np * NP; it += T / 2) {
            const int i = it / NP, j = 8 * (it % NP);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            if (pb >= 0) {
                if constexpr (KV8) {
                    const float s = h2f(a.kv.k_scales[prow + t0 + i]);
                    const u32x2 c = *(const u32x2*)((const int8_t*)a.kv.k + (prow + t0 + i) * D + j);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = (float)(int8_t)((e < 4 ? c.x : c.y) >> (8 * (e & 3))) * s;
                } else {
                    unpack8(*(const u32x4*)((const uint16_t*)a.kv.k + (prow + t0 + i) * D + j), x);
                }
            }
            store(a.k_out, i, j, x);
        }
    }
}

int64_t max_blocks(const fp_chunk& c) { return blocks_before(c.n_rows, c.n_seqs); }

}  // namespace

hipError_t launch_kv_append(const KvAppendArgs& a, bool f32, hipStream_t st) {
    const int64_t n = (max_blocks(a.chunk) + 7) / 8 * 8 * a.kv.n_kv_heads;
    if (n < 1 || n > MAX_GRID) return hipErrorInvalidValue;
    const bool i8 = a.kv.format == FP_KV_INT8;
    const bool tree = a.parent != nullptr && a.cos_t != nullptr;
#define FP_AP(D, I8, F32)                                                                                          \
    do {                                                                                                           \
        if (tree) FP_LAUNCH((kv_append_paged_kernel<D, I8, F32, true>), dim3((unsigned)n), dim3(T), 0, st, a);     \
        else FP_LAUNCH((kv_append_paged_kernel<D, I8, F32, false>), dim3((unsigned)n), dim3(T), 0, st, a);         \
    } while (0)
#define FP_AP_D(D)                                                                   \
    do {                                                                             \
        if (f32) { if (i8) FP_AP(D, true, true); else FP_AP(D, false, true); }       \
        else { if (i8) FP_AP(D, true, false); else FP_AP(D, false, false); }         \
    } while (0)
    if (a.kv.head_dim == 128) FP_AP_D(128);
    else if (a.kv.head_dim == 64) FP_AP_D(64);
    else return hipErrorInvalidValue;
#undef FP_AP_D
#undef FP_AP
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvReadArgs& a, hipStream_t st) {
    const int64_t n = (max_blocks(a.chunk) + 7) / 8 * 8 * a.kv.n_kv_heads;
    if (n < 1 || n > MAX_GRID) return hipErrorInvalidValue;
    const dim3 grid((unsigned)n);
    const bool i8 = a.kv.format == FP_KV_INT8;
    if (a.kv.head_dim == 128) {
        if (i8) FP_LAUNCH((kv_read_paged_kernel<128, true>), grid, dim3(T), 0, st, a);
        else FP_LAUNCH((kv_read_paged_kernel<128, false>), grid, dim3(T), 0, st, a);
    } else if (a.kv.head_dim == 64) {
        if (i8) FP_LAUNCH((kv_read_paged_kernel<64, true>), grid, dim3(T), 0, st, a);
        else FP_LAUNCH((kv_read_paged_kernel<64, false>), grid, dim3(T), 0, st, a);
    } else {
        return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace fpk
