// Beam search's selection: of the continuations of a group's beams by every id, the n_best of the largest
//     s[b] + z[b, v] - log sum_v exp z[b, v]
// (s the beams' scores so far).  Borders between scores decide, so they are in 64 bits: the sums by the exponentials
// of vocab.h, and a score is one sum of 64-bit numbers.  Bound by reading the logits once and by the 64-bit exponentials.
//   rows_kernel    per (row, block of BV ids): maximum, sum of exponentials, and the block's n_best largest logits in order
//   merge_kernel   per group: the rows' sums, then the best of the blocks' lists
//
// A block's candidates: of 64 groups of its ids (a lane's, of all waves) the n_best-th largest of the groups' maxima is
// at most the n_best-th largest logit, as each of those groups has one as large.  What is not below it, some n_best to 2 n_best
// logits unless many are equal, is collected and ranked by counting.
#include "vocab.h"

namespace fpk {

namespace {

constexpr int NT = 256, NW = NT / 64;
constexpr int EPT = 16, BV = NT * EPT;     // ids per thread and block
constexpr int BEST = 64;                   // the most candidates of a group, and beams
constexpr int CAP = 512;                   // candidates of a block that are ranked at once

struct BeamPart {
    double sum;
    float max;
    int n;                                 // entries of the list
};
struct Cand {
    float z;
    int id;
};

// the larger logit, the lower id among equal ones
__device__ __forceinline__ bool before(float za, int ia, float zb, int ib) { return za > zb || (za == zb && ia < ib); }

int blocks_of(int V) { return (V + BV - 1) / BV; }

__global__ void __launch_bounds__(NT) rows_kernel(BeamArgs a, BeamPart* __restrict__ parts, Cand* __restrict__ lists) {
    __shared__ double tab[NT], sd[NW];
    __shared__ float gm[NW][64], cz[CAP];
    __shared__ int ci[CAP], count, tally[2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, K = a.n_best;
    const int64_t row = blockIdx.y, at = row * gridDim.x + blockIdx.x;
    if (a.done != nullptr && a.done[row]) return;
    exp_table(tab);
    const int v0 = blockIdx.x * BV + tid;
    const float* z = a.logits + row * a.row_stride;
    float x[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) x[i] = v0 + NT * i < a.V ? z[v0 + NT * i] : -INFINITY;
    float mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
        x[i] = no_nan(x[i]);
        mine = fmaxf(mine, x[i]);
    }
    gm[w][lane] = mine;
    if (tid == 0) count = 0;
    __syncthreads();
    float grp = gm[0][lane];
#pragma unroll
    for (int j = 1; j < NW; ++j) grp = fmaxf(grp, gm[j][lane]);
    const float m = wave_max(grp);
    if (!(m > -INFINITY)) {                // nothing here
        if (tid == 0) parts[at] = BeamPart{0.0, m, 0};
        return;
    }
    // rank of the lane's group among the 64; the K-th largest maximum
    int rank = 0;
    for (int j = 0; j < 64; ++j) {
        const float o = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(grp), j));
        rank += before(o, j, grp, lane) ? 1 : 0;
    }
    const uint64_t kth = __ballot(rank == K - 1);
    float tau = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(grp), __builtin_ctzll(kth)));
    auto collect = [&](bool equal) {
#pragma unroll
        for (int i = 0; i < EPT; ++i)
            if (x[i] > -INFINITY && (equal ? x[i] >= tau : x[i] > tau)) {
                const int c = atomicAdd(&count, 1);
                if (c < CAP) {
                    cz[c] = x[i];
                    ci[c] = v0 + NT * i;
                }
            }
    };
    collect(true);
    __syncthreads();
    int n = count;
    if (n > CAP) {
        // Many equal ones (or an order that fills few lanes): the K-th largest logit itself by bisection of its bits, those
        // above it, fewer than K, and then of the equal ones the lowest ids.
        auto order = [](float f) {
            const uint32_t u = __float_as_uint(f);
            return u & 0x80000000u ? ~u : u | 0x80000000u;
        };
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = t | 1u << bit;
            int k = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) k += __popcll(__ballot(order(x[i]) >= c));
            if (tid == 0) tally[bit & 1] = 0;
            __syncthreads();
            if (lane == 0) atomicAdd(&tally[bit & 1], k);
            __syncthreads();
            if (tally[bit & 1] >= K) t = c;
        }
        tau = __uint_as_float(t & 0x80000000u ? t & 0x7FFFFFFFu : ~t);
        if (tid == 0) count = 0;
        __syncthreads();
        collect(false);
        __syncthreads();
        n = count;
#pragma unroll
        for (int i = 0; i < EPT; ++i) {    // ids of step i come before those of step i + 1, a lower wave's before a higher's
            const bool eq = x[i] == tau && tau > -INFINITY;
            const uint64_t b = __ballot(eq);
            if (lane == 0) gm[0][w] = __uint_as_float((uint32_t)__popcll(b));
            __syncthreads();
            int c = n, all = 0;
            for (int j = 0; j < NW; ++j) {
                const int k = (int)__float_as_uint(gm[0][j]);
                c += j < w ? k : 0;
                all += k;
            }
            c += __popcll(b & ((1ull << lane) - 1));
            if (eq && c < K) {
                cz[c] = x[i];
                ci[c] = v0 + NT * i;
            }
            n = min(n + all, K);
            __syncthreads();
        }
    }
    for (int j = tid; j < n; j += NT) {
        const float zj = cz[j];
        const int ij = ci[j];
        int r = 0;
        for (int o = 0; o < n; ++o) r += before(cz[o], ci[o], zj, ij) ? 1 : 0;
        if (r < K) lists[at * K + r] = Cand{zj, ij};
    }
    double s = 0.0;
    if (m < INFINITY) {
        const double md = m;
#pragma unroll
        for (int i = 0; i < EPT; ++i) s += weight_below(x[i], md, 1.44269504088896340736, tab);
    } else {
        int k = 0;
#pragma unroll
        for (int i = 0; i < EPT; ++i) k += x[i] == m ? 1 : 0;
        s = k;
    }
    s = wave_sum_d(s);
    if (lane == 0) sd[w] = s;
    __syncthreads();
    if (tid == 0) parts[at] = BeamPart{(sd[0] + sd[1]) + (sd[2] + sd[3]), m, min(n, K)};
}

// ---- merge.  A workgroup per group.
constexpr int MT = 1024;
constexpr int ENT = 1024;                  // entries that are ranked at once
struct Entry {
    double s;
    float z;
    uint32_t at;               // beam, id
};
// The larger score; of equal ones the lower beam, in it the larger logit, then the lower id.
__device__ __forceinline__ bool better(const Entry& x, const Entry& y) {
    if (x.s != y.s) return x.s > y.s;
    if (x.at >> 20 != y.at >> 20) return x.at >> 20 < y.at >> 20;
    return before(x.z, x.at & 0xFFFFF, y.z, y.at & 0xFFFFF);
}

__global__ void __launch_bounds__(MT) merge_kernel(BeamArgs a, int nb, const BeamPart* __restrict__ parts, const Cand* __restrict__ lists) {
    __shared__ Entry ent[ENT];
    __shared__ double tab[256], base[BEST], head[MT], cut;
    __shared__ float top[BEST];
    __shared__ int count, won[MT / 64];
    __shared__ uint8_t taken[BEST * ((1 << 20) / BV)];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = blockIdx.x, W = a.n_beams, K = a.n_best;
    const int64_t row0 = (int64_t)g * W;
    if (tid < 256) exp_table(tab);
    if (tid == 0) {
        count = 0;
        cut = -INFINITY;
    }
    __syncthreads();
    // a row's sum: base + (z - m) is the score of a continuation (z - m first: of a row whose logits all are the type's
    // lowest value it is zero, and the sum's logarithm is not lost)
    for (int b = w; b < W; b += MT / 64) {
        const float sc = a.scores[row0 + b];
        const bool done = a.done != nullptr && a.done[row0 + b];
        float m = -INFINITY;
        double s = 0.0;
        if (!done) {
            const BeamPart* p = parts + (row0 + b) * nb;
            for (int j = lane; j < nb; j += 64) m = fmaxf(m, p[j].max);
            m = wave_max(m);
            if (m > -INFINITY)
                for (int j = lane; j < nb; j += 64) s += p[j].sum * weight(p[j].max, m, 1.44269504088896340736, tab);
            s = wave_sum_d(s);
        }
        if (lane == 0) {
            // a beam of no score, or without any logit, has no continuation
            const bool live = sc > -INFINITY && (done || m > -INFINITY);
            base[b] = !live ? -INFINITY : done ? (double)sc : (double)sc - log(s);
            top[b] = m;
        }
    }
    __syncthreads();
    // Entry r of list l (a row's blocks one after another; a finished beam has one list of itself).
    const int L = W * nb;
    auto entry = [&](int l, int r, Entry& e) {
        const int b = l / nb;
        if (!(base[b] > -INFINITY)) return false;
        if (a.done != nullptr && a.done[row0 + b]) {
            e = Entry{base[b], 0.f, (uint32_t)b << 20};
            return l % nb == 0 && r == 0;
        }
        const int64_t at = row0 * nb + l;
        if (r >= parts[at].n) return false;
        const Cand c = lists[at * K + r];
        if (top[b] == INFINITY && c.z < INFINITY) return false;       // infinite logits share the whole
        e = Entry{base[b] + (top[b] == INFINITY ? 0.0 : (double)c.z - (double)top[b]), c.z, (uint32_t)b << 20 | (uint32_t)c.id};
        return true;
    };
    auto emit = [&](int r, const Entry& e) {
        const int b = e.at >> 20;
        const bool was = a.done != nullptr && a.done[row0 + b];
        const int id = was ? a.pad : (int)(e.at & 0xFFFFF);
        const int64_t o = (int64_t)g * K + r;
        a.out_scores[o] = (float)e.s;
        a.out_parent[o] = b;
        a.out_ids[o] = id;
        if (a.out_done != nullptr) a.out_done[o] = was || id == a.eos;
    };
    // The K-th largest of the threads' best heads is at most the K-th largest entry.
    double best = -INFINITY;
    for (int l = tid; l < L; l += MT) {
        Entry e;
        if (entry(l, 0, e)) best = fmax(best, e.s);
    }
    head[tid] = best;
    __syncthreads();
    const int H = min(L, MT);
    if (H >= K && tid < H) {
        int r = 0;
        for (int j = 0; j < H; ++j) r += head[j] > best || (head[j] == best && j < tid) ? 1 : 0;
        if (r == K - 1) cut = best;
    }
    __syncthreads();
    for (int l = tid; l < L; l += MT) {
        Entry e;
        for (int r = 0; r < K && entry(l, r, e) && e.s >= cut; ++r) {
            const int i = atomicAdd(&count, 1);
            if (i < ENT) ent[i] = e;
        }
    }
    __syncthreads();
    int n = count;
    if (n <= ENT) {
        for (int i = tid; i < n; i += MT) {
            const Entry e = ent[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += better(ent[j], e) ? 1 : 0;
            if (r < K) emit(r, e);
        }
    } else {
        // Many equal scores, or few long lists: the lists are merged head by head.
        for (int l = tid; l < L; l += MT) taken[l] = 0;
        Entry mine;
        int from;
        auto heads = [&]() {               // the best head of the thread's lists
            from = -1;
            for (int l = tid; l < L; l += MT) {
                Entry e;
                if (taken[l] < K && entry(l, taken[l], e) && (from < 0 || better(e, mine))) {
                    mine = e;
                    from = l;
                }
            }
        };
        heads();
        for (n = 0; n < K; ++n) {
            Entry e = mine;
            int l = from;
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) {
                const Entry y = {__shfl_xor(e.s, o, 64), __shfl_xor(e.z, o, 64), __shfl_xor(e.at, o, 64)};
                const int yl = __shfl_xor(l, o, 64);
                if (yl >= 0 && (l < 0 || better(y, e))) {
                    e = y;
                    l = yl;
                }
            }
            __syncthreads();
            if (lane == 0) {
                ent[w] = e;
                won[w] = l;
            }
            __syncthreads();
            e = ent[0];
            l = won[0];
            for (int j = 1; j < MT / 64; ++j)
                if (won[j] >= 0 && (l < 0 || better(ent[j], e))) {
                    e = ent[j];
                    l = won[j];
                }
            if (l < 0) break;
            if (tid == 0) emit(n, e);
            if (l == from) {
                ++taken[l];
                heads();
            }
        }
    }
    for (int r = min(n, K) + tid; r < K; r += MT) {
        const int64_t o = (int64_t)g * K + r;
        a.out_scores[o] = -INFINITY;
        a.out_parent[o] = -1;
        a.out_ids[o] = -1;
        if (a.out_done != nullptr) a.out_done[o] = 0;
    }
}

}  // namespace

size_t beam_ws_bytes(int n_rows, int n_best, int V) {
    return (size_t)n_rows * blocks_of(V) * (sizeof(BeamPart) + n_best * sizeof(Cand));
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t st) {
    const int nb = blocks_of(a.V), rows = a.n_groups * a.n_beams;
    BeamPart* parts = (BeamPart*)a.ws;
    Cand* lists = (Cand*)(parts + (size_t)rows * nb);
    FP_LAUNCH(rows_kernel, dim3(nb, rows), dim3(NT), 0, st, a, parts, lists);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    FP_LAUNCH(merge_kernel, dim3(a.n_groups), dim3(MT), 0, st, a, nb, parts, lists);
    return hipGetLastError();
}

}  // namespace fpk
