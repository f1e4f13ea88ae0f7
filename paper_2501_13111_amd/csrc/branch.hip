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
// are one or two cache lines.  Bound by latency: lengths and path, pages, elements, one after another.  Paths of up to 7 of 40 sequences
// on 8 heads of 128, four int8 layers: 6.1 us in a graph of them, 6.9 by a kernel trace (5 MB in, 5 out); one path of 3 on 32 heads, two bf16
// layers: 3.9 and 4.7.
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
        // lengths and path together, then both pages of a move: positions below max_len are inside the table
        const int src = tid < a.path_stride ? a.path[(int64_t)b * a.path_stride + tid] : -1;
        const int keep = min(a.n_keep[b], sq.n), bpp = kv.page_size / VT_BLK;
        const bool moves = tid < keep && src >= 0 && src < sq.n && src != tid;
        const int bt = (sq.ctx + (moves ? tid : 0)) / VT_BLK, bs = (sq.ctx + (moves ? src : 0)) / VT_BLK;
        const int* row = a.chunk.table + (int64_t)b * a.chunk.table_stride;
        const int gt = moves ? row[bt / bpp] : -1, gs = moves ? row[bs / bpp] : -1;
        const int pt = gt >= 0 && gt < kv.n_pages ? (gt * kv.n_kv_heads + kvh) * bpp + bt % bpp : -1;
        const int ps = gs >= 0 && gs < kv.n_pages ? (gs * kv.n_kv_heads + kvh) * bpp + bs % bpp : -1;
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
    const int n = __builtin_amdgcn_readfirstlane(count);
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
    // eight at a time: most paths are short (in a graph 1.0 and 0.7 us less than if every turn asks for itself)
#pragma unroll
    for (int x0 = 0; x0 < VX; x0 += 8) {
        if (T * x0 >= n * D) break;
#pragma unroll
        for (int x = x0; x < x0 + 8; ++x) {
            const int it = tid + T * x;
            v[x] = 0;
            if (it < n * D) {
                const int i = it % n, d = it / n;
                if (from[i] >= 0) v[x] = ((const V*)kv.v)[((int64_t)from[i] * D + d) * VT_BLK + vt_slot(at[i] >> 8)];
            }
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
    for (int x0 = 0; x0 < VX; x0 += 8) {
        if (T * x0 >= n * D) break;
#pragma unroll
        for (int x = x0; x < x0 + 8; ++x) {
            const int it = tid + T * x;
            if (it < n * D) {
                const int i = it % n, d = it / n;
                ((V*)kv.v)[((int64_t)to[i] * D + d) * VT_BLK + vt_slot(at[i] & 255)] = v[x];
            }
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

// Sixty-four columns' worth of lanes of group g's table, by one wave: full pages from the beam that a beam goes on from, the
// last one from its giver, those behind it its own.  All entries are read before any is written: table_out may be the table.
__device__ __forceinline__ void table_wave(const ReorderArgs& a, int page_size, const BeamMap& m, int g, int chunk, int cols) {
    const int W = a.n_beams, lane = threadIdx.x & 63;
    const int len = group_len(a, g), full = len / page_size, part = len % page_size != 0;
    const int w = lane / cols, c = chunk * cols + lane % cols;
    const int from = __shfl(m.from, w, 64), giver = __shfl(m.giver, w, 64);
    const bool on = w < W && c < a.width;
    const int64_t row = (int64_t)g * W;
    const int own = on ? a.table[(row + w) * a.table_stride + c] : -1;
    const int up = __shfl(own, from * cols + lane % cols, 64), last = __shfl(own, giver * cols + lane % cols, 64);
    const int v = c < full ? up : c == full && part ? last : own;
    if (on && (v != own || a.table_out != a.table)) a.table_out[(row + w) * a.out_stride + c] = v;
}
// Columns of a wave: 64 / n_beams to a power of two.
__host__ __device__ __forceinline__ int table_cols(int n_beams) {
    int cols = 64;
    while (cols * n_beams > 64) cols >>= 1;
    return cols;
}

__global__ void __launch_bounds__(64) beam_table_kernel(int page_size, ReorderArgs a) {
    const BeamMap m = beam_map(a, blockIdx.y);
    table_wave(a, page_size, m, blockIdx.y, blockIdx.x, table_cols(a.n_beams));
}

// The partly filled last page of the beam that an extra beam goes on from, copied into its own, and, as one layer more, the table if
// that goes elsewhere.  The workgroups of a (group, layer) take shares of its copies in turn: 32-position blocks of keys or of
// values, eight 16-byte loads a thread in flight.  Whole blocks: what lies behind the last position may be anything.  Parents, table
// and data are a chain of three latencies, so there are no more workgroups than run at a time.  16 groups of 8 beams, 4 layers, int8,
// 121 MB in random pages: 26 us, 4.6 TB/s (one workgroup for each pair of blocks that might have to be copied 41; the eight loads
// under a mask, each waiting for the one before, 58).
template <int D, bool KV8>
__global__ void __launch_bounds__(T) beam_copy_kernel(KvSet kvs, ReorderArgs a) {
    constexpr int N = VT_BLK * D * (KV8 ? 1 : 2) / 16;     // 16-byte pieces of a block of keys or of values
    constexpr int TPB = N < T ? N : T, PX = N / TPB;       // threads of a block, pieces of a thread
    constexpr int SIDE = T / TPB, X = 8 / PX;              // blocks side by side, and after each other
    const int tid = threadIdx.x, ps = kvs.kv[0].page_size, bpp = ps / VT_BLK, g = blockIdx.y;
    const int len = group_len(a, g), col = len / ps;
    const BeamMap m = beam_map(a, g);
    if ((int)blockIdx.z == kvs.n) {
        const int cols = table_cols(a.n_beams);
        for (int c = blockIdx.x * (T / 64) + (tid >> 6); c * cols < a.width; c += gridDim.x * (T / 64)) table_wave(a, ps, m, g, c, cols);
        return;
    }
    const fp_paged_kv& kv = kvs.kv[blockIdx.z];
    const int blocks = (len % ps + VT_BLK - 1) / VT_BLK, all = 2 * blocks * kv.n_kv_heads;      // of keys and values, of a copy
    const int shares = (all + X * SIDE - 1) / (X * SIDE), items = __popcll(m.extra) * shares;
    if ((int)blockIdx.x >= items || col >= a.width) return;
    // lane b: the pages of beam b's copy
    const int lane = tid & 63;
    const int* t = a.table + (int64_t)g * a.n_beams * a.table_stride + col;
    int from_page = -1, to_page = -1;
    if (m.extra >> lane & 1) {
        from_page = t[(int64_t)m.from * a.table_stride];
        to_page = t[(int64_t)m.giver * a.table_stride];
    }
    for (int it = blockIdx.x; it < items; it += gridDim.x) {
        uint64_t x = m.extra;
        for (int i = it / shares; i > 0; --i) x &= x - 1;
        const int b = __builtin_ctzll(x), i0 = it % shares * (X * SIDE);
        const int src = __builtin_amdgcn_readlane(from_page, b), dst = __builtin_amdgcn_readlane(to_page, b);
        if (dst < 0 || dst >= kv.n_pages) continue;
        const bool ok = src >= 0 && src < kv.n_pages;      // a missing page reads as zeros
        const int64_t per = (int64_t)kv.n_kv_heads * bpp, from = ok ? src * per : 0, to = dst * per;      // in blocks
        // Block i of the copy, of keys if even: its data and scales at `page` of the pool, nothing past the last.  (Loads and stores
        // past a resource's end do nothing: no branch around one, at whose end the loads before it would be waited for.)
        auto data = [&](int i, int64_t page, bool on) {
            const int64_t at = page + (i >> 1) / blocks * bpp + (i >> 1) % blocks;
            return buf_rsrc((const u32x4*)(i & 1 ? kv.v : kv.k) + (on ? at * N : 0), on ? 16 * N : 0);
        };
        auto scale = [&](int i, int64_t page, bool on) {
            const int64_t at = page + (i >> 1) / blocks * bpp + (i >> 1) % blocks;
            return buf_rsrc((i & 1 ? kv.v_scales : kv.k_scales) + (on ? at * VT_BLK : 0), on ? 2 * VT_BLK : 0);
        };
        const int i1 = __builtin_amdgcn_readfirstlane(i0 + tid / TPB), q = tid % TPB;
        u32x4 v[X][PX], sc[X];
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const int i = i1 + k * SIDE;
            const auto r = data(i, from, ok && i < all);
#pragma unroll
            for (int y = 0; y < PX; ++y) v[k][y] = __builtin_amdgcn_raw_buffer_load_b128(r, 16 * (q + TPB * y), 0, 0);
            if (KV8) sc[k] = __builtin_amdgcn_raw_buffer_load_b128(scale(i, from, ok && i < all), 16 * q, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < X; ++k) {
            const int i = i1 + k * SIDE;
            const auto r = data(i, to, i < all);
#pragma unroll
            for (int y = 0; y < PX; ++y) __builtin_amdgcn_raw_buffer_store_b128(v[k][y], r, 16 * (q + TPB * y), 0, 0);
            if (KV8) __builtin_amdgcn_raw_buffer_store_b128(sc[k], scale(i, to, i < all), 16 * q, 0, 0);
        }
    }
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

hipError_t launch_beam_copy(const KvSet& kvs, const ReorderArgs& a, bool table, hipStream_t st) {
    const fp_paged_kv& kv = kvs.kv[0];
    if (a.n_beams < 2) return hipErrorInvalidValue;
    // eight blocks of 4 KB, four of 8, and so on, are what a workgroup takes at a time
    const int64_t share = 32768 / (VT_BLK * kv.head_dim * (kv.format == FP_KV_INT8 ? 1 : 2));
    const int64_t most = (2ll * kv.n_kv_heads * (kv.page_size / VT_BLK) + share - 1) / share * (a.n_beams - 1);
    const int64_t x = std::min<int64_t>(most, std::max<int64_t>(1, 1280 / ((int64_t)a.n_groups * kvs.n)));
    FP_SET(beam_copy_kernel, dim3((unsigned)x, a.n_groups, kvs.n + (table ? 1 : 0)), a);
    return hipGetLastError();
}

hipError_t launch_beam_table(int page_size, const ReorderArgs& a, hipStream_t st) {
    const int cols = table_cols(a.n_beams);
    FP_LAUNCH(beam_table_kernel, dim3((a.width + cols - 1) / cols, a.n_groups), dim3(64), 0, st, page_size, a);
    return hipGetLastError();
}

}  // namespace fpk
