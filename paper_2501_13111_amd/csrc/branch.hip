// Positions of a paged cache that change places when a sequence goes on in one of several ways, in all layers at once:
// the accepted path of a drafted tree moves to the front of its nodes, and beams go on from other beams' caches.
#include <algorithm>
#include <type_traits>

#include "tree.h"

namespace fpk {

namespace {

constexpr int T = 256;

// Position j of sequence b's path (node path[b][j]) moves to position ctx + j, keys, values and scales, of one kv head
// of one layer per workgroup.  Every element is read before any is written, so a path may be any list of nodes.
// Elements of a value lie 32 slots apart: neighbouring threads take the positions of one dim, whose slots
// are one or two cache lines.
template <int D, bool KV8>
__global__ void __launch_bounds__(T) kv_keep_kernel(KvSet kvs, KvKeepArgs a) {
    constexpr int ES = KV8 ? 1 : 2, NP = D * ES / 16;      // 16-byte pieces of a key
    constexpr int KX = TREE_MAX * NP / T, VX = TREE_MAX * D / T;
    using V = typename std::conditional<KV8, uint8_t, uint16_t>::type;
    __shared__ int from[TREE_MAX], to[TREE_MAX], at[TREE_MAX];      // pool positions of the moves; their place in the path
    __shared__ int count;
    const fp_paged_kv& kv = kvs.kv[blockIdx.y];
    const int tid = threadIdx.x, b = blockIdx.x / kv.n_kv_heads, kvh = blockIdx.x % kv.n_kv_heads;
    const Seq sq = load_seq(a.chunk, b);
    if (tid < 64) {
        const int keep = min(min(a.n_keep[b], a.path_stride), sq.n);
        const int src = tid < keep ? a.path[(int64_t)b * a.path_stride + tid] : -1;
        const bool moves = src >= 0 && src < sq.n && src != tid;
        int pt = -1, ps = -1;
        if (moves) {
            pt = pool_block(kv, a.chunk, b, kvh, (sq.ctx + tid) / VT_BLK);
            ps = pool_block(kv, a.chunk, b, kvh, (sq.ctx + src) / VT_BLK);
        }
        const uint64_t any = __ballot(pt >= 0);
        if (pt >= 0) {
            const int i = __popcll(any & ((1ull << tid) - 1));
            to[i] = pt;
            from[i] = ps;
            at[i] = ((sq.ctx + tid) % VT_BLK) | ((sq.ctx + src) % VT_BLK) << 8;
        }
        if (tid == 0) count = __popcll(any);
    }
    __syncthreads();
    const int n = count;
    u32x4 k[KX];
    V v[VX];
    uint16_t sc = 0;
#pragma unroll
    for (int x = 0; x < KX; ++x) {
        const int it = tid + T * x, i = it / NP;
        k[x] = u32x4{0u, 0u, 0u, 0u};
        if (i < n && from[i] >= 0)
            k[x] = *(const u32x4*)((const char*)kv.k + ((int64_t)from[i] * VT_BLK + (at[i] >> 8)) * D * ES + 16 * (it % NP));
    }
#pragma unroll
    for (int x = 0; x < VX; ++x) {
        const int it = tid + T * x;
        v[x] = 0;
        if (it < n * D) {
            const int i = it % n, d = it / n;
            if (from[i] >= 0) v[x] = ((const V*)kv.v)[((int64_t)from[i] * D + d) * VT_BLK + vt_slot(at[i] >> 8)];
        }
    }
    const int si = tid & 63;                               // KV8: threads below 64 key scales, below 128 value scales
    uint16_t* const scales = tid < 64 ? kv.k_scales : kv.v_scales;
    if (KV8 && tid < 128 && si < n && from[si] >= 0) sc = scales[(int64_t)from[si] * VT_BLK + (at[si] >> 8)];
    __syncthreads();
#pragma unroll
    for (int x = 0; x < KX; ++x) {
        const int it = tid + T * x, i = it / NP;
        if (i < n) *(u32x4*)((char*)kv.k + ((int64_t)to[i] * VT_BLK + (at[i] & 255)) * D * ES + 16 * (it % NP)) = k[x];
    }
#pragma unroll
    for (int x = 0; x < VX; ++x) {
        const int it = tid + T * x;
        if (it < n * D) {
            const int i = it % n, d = it / n;
            ((V*)kv.v)[((int64_t)to[i] * D + d) * VT_BLK + vt_slot(at[i] & 255)] = v[x];
        }
    }
    if (KV8 && tid < 128 && si < n) scales[(int64_t)to[si] * VT_BLK + (at[si] & 255)] = sc;
}

// Who goes on from whom in a group of up to 64 beams; lane b has beam b.  The first beam that goes on from a beam keeps
// its last page, the others take the pages of the beams that none goes on from, in order: there are as many.
struct BeamMap {
    int from;                  // the beam that lane b goes on from (a parent out of range: itself)
    uint64_t extra, free;      // beams that are not the first of theirs; beams that none goes on from
    int giver;                 // the beam whose last page lane b's beam has from now on
};
__device__ __forceinline__ BeamMap beam_map(const ReorderArgs& a, int g) {
    const int lane = threadIdx.x & 63, W = a.n_beams;
    BeamMap m;
    m.from = lane < W ? a.parent[(int64_t)g * W + lane] : 0;
    if (lane < W && (m.from < 0 || m.from >= W)) m.from = lane;
    const uint64_t beams = W == 64 ? ~0ull : (1ull << W) - 1, below = (1ull << lane) - 1;
    uint64_t same = beams, mine = beams;                   // beams that go on from mine's; that go on from beam `lane`
#pragma unroll
    for (int k = 0; k < 6; ++k) {
        const uint64_t one = __ballot(m.from >> k & 1);
        same &= m.from >> k & 1 ? one : ~one;
        mine &= lane >> k & 1 ? one : ~one;
    }
    const bool extra = lane < W && (same & below) != 0;
    m.extra = __ballot(extra);
    m.free = __ballot(lane < W && mine == 0);
    // lane of the free beam of my rank
    m.giver = m.from;
    const int rank = __popcll(m.extra & below);
    uint64_t f = m.free;
    for (int i = 0; f != 0; ++i, f &= f - 1)
        if (extra && rank == i) m.giver = __builtin_ctzll(f);
    return m;
}
// The group's positions: those of its first beam.
__device__ __forceinline__ int group_len(const ReorderArgs& a, int g) { return max(a.ctx_len[(int64_t)g * a.n_beams], 0); }

// The partly filled last page of the beam that an extra beam goes on from, copied into its own: workgroups per (extra
// beam, layer) share its 32-position blocks.  Whole blocks: what lies behind the last position may be anything.
template <int D, bool KV8>
__global__ void __launch_bounds__(T) beam_copy_kernel(KvSet kvs, ReorderArgs a) {
    constexpr int N = VT_BLK * D * (KV8 ? 1 : 2) / 16;     // 16-byte pieces of a block of keys, and of values
    constexpr int X = (N + T - 1) / T;
    const fp_paged_kv& kv = kvs.kv[blockIdx.z];
    const int bpp = kv.page_size / VT_BLK, tid = threadIdx.x;
    const int g = blockIdx.y / (a.n_beams - 1), e = blockIdx.y % (a.n_beams - 1);
    const int len = group_len(a, g), col = len / kv.page_size, blocks = (len % kv.page_size + VT_BLK - 1) / VT_BLK;
    if ((int)blockIdx.x >= blocks * kv.n_kv_heads || col >= a.width) return;
    const BeamMap m = beam_map(a, g);
    if (e >= __popcll(m.extra)) return;
    uint64_t x = m.extra;
    for (int i = 0; i < e; ++i) x &= x - 1;
    const int b = __builtin_ctzll(x);
    const int* t = a.table + (int64_t)g * a.n_beams * a.table_stride + col;
    const int src = t[(int64_t)__builtin_amdgcn_readlane(m.from, b) * a.table_stride];
    const int dst = t[(int64_t)__builtin_amdgcn_readlane(m.giver, b) * a.table_stride];
    if (dst < 0 || dst >= kv.n_pages) return;
    const bool ok = src >= 0 && src < kv.n_pages;          // a missing page reads as zeros
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (int u = blockIdx.x; u < blocks * kv.n_kv_heads; u += gridDim.x) {
        const int in = u / blocks * bpp + u % blocks;      // of the page's blocks
        const int64_t per = (int64_t)kv.n_kv_heads * bpp, from = (ok ? src * per : 0) + in, to = dst * per + in;
        const u32x4 *ks = (const u32x4*)kv.k + from * N, *vs = (const u32x4*)kv.v + from * N;
        u32x4 *kd = (u32x4*)kv.k + to * N, *vd = (u32x4*)kv.v + to * N;
        u32x4 k[X], v[X];
#pragma unroll
        for (int i = 0; i < X; ++i) {
            const int it = tid + T * i;
            k[i] = ok && it < N ? ks[it] : zero;
            v[i] = ok && it < N ? vs[it] : zero;
        }
#pragma unroll
        for (int i = 0; i < X; ++i) {
            const int it = tid + T * i;
            if (it < N) {
                kd[it] = k[i];
                vd[it] = v[i];
            }
        }
        if (KV8 && tid < 2 * VT_BLK / 8) {                 // scales: 64 bytes each
            uint16_t* s = tid < VT_BLK / 8 ? kv.k_scales : kv.v_scales;
            const int i = tid % (VT_BLK / 8);
            ((u32x4*)s)[to * (VT_BLK / 8) + i] = ok ? ((const u32x4*)s)[from * (VT_BLK / 8) + i] : zero;
        }
    }
}

// The table: full pages from the beam that a beam goes on from, the last one from its giver, those behind it its own.
// A wave takes the group's entries of some columns, all read before any is written: table_out may be the table.
__global__ void __launch_bounds__(64) beam_table_kernel(int page_size, ReorderArgs a) {
    const int W = a.n_beams, g = blockIdx.y, lane = threadIdx.x;
    const int len = group_len(a, g), full = len / page_size, part = len % page_size != 0;
    const BeamMap m = beam_map(a, g);
    int cols = 64;                                         // columns of a wave: 64 / W to a power of two
    while (cols * W > 64) cols >>= 1;
    const int w = lane / cols, c = blockIdx.x * cols + lane % cols;
    const int from = __shfl(m.from, w, 64), giver = __shfl(m.giver, w, 64);
    const bool on = w < W && c < a.width;
    const int64_t row = (int64_t)g * W;
    const int own = on ? a.table[(row + w) * a.table_stride + c] : -1;
    const int up = __shfl(own, from * cols + lane % cols, 64), last = __shfl(own, giver * cols + lane % cols, 64);
    const int v = c < full ? up : c == full && part ? last : own;
    if (on && (v != own || a.table_out != a.table)) a.table_out[(row + w) * a.out_stride + c] = v;
}

}  // namespace

#define FP_SET(KERNEL, GRID, ...)                                                                          \
    do {                                                                                                   \
        const bool i8 = kvs.kv[0].format == FP_KV_INT8;                                                    \
        const int D = kvs.kv[0].head_dim;                                                                  \
        if (D == 128 && i8) FP_LAUNCH((KERNEL<128, true>), GRID, dim3(T), 0, st, kvs, __VA_ARGS__);        \
        else if (D == 128) FP_LAUNCH((KERNEL<128, false>), GRID, dim3(T), 0, st, kvs, __VA_ARGS__);        \
        else if (D == 64 && i8) FP_LAUNCH((KERNEL<64, true>), GRID, dim3(T), 0, st, kvs, __VA_ARGS__);     \
        else if (D == 64) FP_LAUNCH((KERNEL<64, false>), GRID, dim3(T), 0, st, kvs, __VA_ARGS__);          \
        else return hipErrorInvalidValue;                                                                  \
    } while (0)

hipError_t launch_kv_keep(const KvSet& kvs, const KvKeepArgs& a, hipStream_t st) {
    const int64_t n = (int64_t)a.chunk.n_seqs * kvs.kv[0].n_kv_heads;
    if (n > MAX_GRID / KV_SET) return hipErrorInvalidValue;
    FP_SET(kv_keep_kernel, dim3((unsigned)n, kvs.n), a);
    return hipGetLastError();
}

hipError_t launch_beam_copy(const KvSet& kvs, const ReorderArgs& a, hipStream_t st) {
    const fp_paged_kv& kv = kvs.kv[0];
    const int64_t y = (int64_t)a.n_groups * (a.n_beams - 1);
    if (y == 0) return hipSuccess;
    if (y > 65535) return hipErrorInvalidValue;
    const int64_t x = std::min<int64_t>((int64_t)kv.n_kv_heads * (kv.page_size / VT_BLK), std::max<int64_t>(8, 16384 / y));
    FP_SET(beam_copy_kernel, dim3((unsigned)x, (unsigned)y, kvs.n), a);
    return hipGetLastError();
}

hipError_t launch_beam_table(int page_size, const ReorderArgs& a, hipStream_t st) {
    int cols = 64;
    while (cols * a.n_beams > 64) cols >>= 1;
    FP_LAUNCH(beam_table_kernel, dim3((a.width + cols - 1) / cols, a.n_groups), dim3(64), 0, st, page_size, a);
    return hipGetLastError();
}

}  // namespace fpk
