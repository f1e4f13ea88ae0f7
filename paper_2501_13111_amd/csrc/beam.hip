// Beam search's selection: of the continuations of a group's beams by every id, the n_best of the largest
//     s[b] + z[b, v] - log sum_v exp z[b, v]
// (s the beams' scores so far).  Borders between scores decide, so they are in 64 bits: the sums by the exponentials
// of vocab.h, and a score is one sum of 64-bit numbers.  Bound by reading the logits once and by the 64-bit exponentials.
//   rows_kernel    per (row, block of BV ids): maximum, sum of exponentials, and the block's n_best largest logits in order
//   merge_kernel   per group: the rows' sums, then the best of the blocks' lists
//
// A block's candidates: of 64 groups of its ids (a lane's, of all waves) the n_best-th largest of the groups' maxima is
// at most the n_best-th largest logit, as each of those groups has one as large.  What is not below it, some n_best to 2 n_best
// logits unless many are equal, is collected and ranked by counting.  The merge bounds its entries by the lists' heads in the same way.
//
// 24 groups of 8 beams over 128000 ids, 16 best, some beams finished: 25.7 us for the rows (78.5 MB of those that are not, 3.1 TB/s), 7.8 for the
// merge.  One group of 4 over 32000: 5.1 + 5.4, both chains of latencies.
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

int blocks_of(int V) { return (V + BV - 1) / BV; }

// Floats in an order that unsigned numbers have (no NaN), and back.
__device__ __forceinline__ uint32_t order(float f) {
    const uint32_t u = __float_as_uint(f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unorder(uint32_t t) { return __uint_as_float(t & 0x80000000u ? t & 0x7FFFFFFFu : ~t); }

// Candidates as numbers in their order: the larger logit, of equal ones (0 and -0 too) the lower id.
__device__ __forceinline__ uint64_t cand_key(float z, uint32_t id) { return (uint64_t)order(z + 0.f) << 32 | ~id; }

// How many of n keys are larger (8 reads at a time: alone, each would wait for the one before).
template <class T>
__device__ __forceinline__ int rank_of(const T* keys, int n, const T& me) {
    int r = 0, o = 0;
    for (; o + 8 <= n; o += 8) {
        T k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) k[j] = keys[o + j];
#pragma unroll
        for (int j = 0; j < 8; ++j) r += me < k[j] ? 1 : 0;
    }
    for (; o < n; ++o) r += me < keys[o] ? 1 : 0;
    return r;
}

// A number that at least k of the wave's lanes are not below: the k-th largest with the bits under `low` cleared.
__device__ __forceinline__ uint32_t kth_largest(uint32_t key, int k, int low) {
    uint32_t t = 0;
    for (int bit = 31; bit >= low; --bit) {
        const uint32_t c = t | 1u << bit;
        if (__popcll(__ballot(key >= c)) >= k) t = c;
    }
    return t;
}

// exp(z - m) from a table whose entries lie in different banks of LDS.  NaN and -inf give 2^-900.
__device__ __forceinline__ double exp_near(float z, double m, const double* tab) {
    return exp2_series<32>(fmax(((double)z - m) * 1.44269504088896340736, -900.0), tab);
}

__global__ void __launch_bounds__(NT, 8) rows_kernel(BeamArgs a, BeamPart* __restrict__ parts, Cand* __restrict__ lists) {
    __shared__ double tab[32], sd[NW];
    __shared__ float gm[NW][64];
    __shared__ uint64_t cand[CAP];
    __shared__ int count, tally[2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, K = a.n_best;
    const int64_t row = blockIdx.y, at = row * gridDim.x + blockIdx.x;
    if (a.done != nullptr && a.done[row]) return;
    const int v0 = blockIdx.x * BV + tid;
    // past the row's end a load gives zeros
    const int here = min(a.V - (int)blockIdx.x * BV, BV);
    const auto z = buf_rsrc(a.logits + row * a.row_stride + blockIdx.x * BV, 4 * here);
    float x[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) x[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(z, 4 * tid, 4 * NT * i, 0));
    if (here < BV) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) x[i] = tid + NT * i < here ? x[i] : -INFINITY;
    }
    exp_table(tab);
    float mine = -INFINITY;                // (NaN is no maximum, and passes no comparison below)
#pragma unroll
    for (int i = 0; i < EPT; ++i) mine = fmaxf(mine, x[i]);
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
    float tau = fmaxf(unorder(kth_largest(order(grp), K, 14)), -INFINITY);       // (NaN: fewer than K groups have any)
    auto collect = [&](auto passes) {
#pragma unroll
        for (int i = 0; i < EPT; ++i)
            if (x[i] > -INFINITY && passes(x[i])) {
                const int c = atomicAdd(&count, 1);
                if (c < CAP) cand[c] = cand_key(x[i], v0 + NT * i);
            }
    };
    if (mine >= tau) collect([&](float v) { return v >= tau; });
    double s = 0.0;
    if (m < INFINITY) {
        const double md = m;
#pragma unroll
        for (int i = 0; i < EPT; ++i) s += exp_near(x[i], md, tab);
    } else {
        int k = 0;
#pragma unroll
        for (int i = 0; i < EPT; ++i) k += x[i] == m ? 1 : 0;
        s = k;
    }
    s = wave_sum_d(s);
    if (lane == 0) sd[w] = s;
    __syncthreads();
    int n = count;
    if (n > CAP) {
        // Many equal ones (or an order that fills few lanes): the K-th largest logit itself by bisection of its bits, those
        // above it, fewer than K, and then of the equal ones the lowest ids.
        uint32_t t = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = t | 1u << bit;
            int k = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) k += __popcll(__ballot(order(no_nan(x[i])) >= c));
            if (tid == 0) tally[bit & 1] = 0;
            __syncthreads();
            if (lane == 0) atomicAdd(&tally[bit & 1], k);
            __syncthreads();
            if (tally[bit & 1] >= K) t = c;
        }
        tau = unorder(t);
        if (tid == 0) count = 0;
        __syncthreads();
        collect([&](float v) { return v > tau; });
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
            if (eq && c < K) cand[c] = cand_key(x[i], v0 + NT * i);
            n = min(n + all, K);
            __syncthreads();
        }
    }
    if (tid == 0) parts[at] = BeamPart{(sd[0] + sd[1]) + (sd[2] + sd[3]), m, min(n, K)};
    for (int j = tid; j < n; j += NT) {
        const uint64_t me = cand[j];
        const int r = rank_of(cand, n, me);
        if (r < K) lists[at * K + r] = Cand{unorder(me >> 32), (int)~(uint32_t)me};
    }
}

// ---- merge.  A workgroup of MT threads per group.
constexpr int ENT = 1024;                  // entries that are ranked at once
// A continuation as a number in their order: the larger score; of equal ones the lower beam, in it the larger logit, then the
// lower id.
struct Entry {
    uint64_t score, at;
    __device__ __forceinline__ bool operator<(const Entry& o) const { return score < o.score || (score == o.score && at < o.at); }
};
__device__ __forceinline__ uint64_t order(double v) {
    const uint64_t u = __double_as_longlong(v);
    return u ^ ((uint64_t)((int64_t)u >> 63) | 1ull << 63);
}
__device__ __forceinline__ double unorder(uint64_t t) { return __longlong_as_double(t >> 63 ? t & ~(1ull << 63) : ~t); }
__device__ __forceinline__ Entry make_entry(double s, int b, float z, int id) {
    return Entry{order(s + 0.0), (uint64_t)(BEST - 1 - b) << 52 | (uint64_t)order(z + 0.f) << 20 | (uint64_t)(0xFFFFF - id)};
}

// A chain of latencies: the lists' parts and heads are loaded together, and then all entries of the lists whose heads pass.
template <int MT>
__global__ void __launch_bounds__(MT) merge_kernel(BeamArgs a, int nb, const BeamPart* __restrict__ parts, const Cand* __restrict__ lists) {
    __shared__ Entry ent[ENT];
    __shared__ double tab[EXP_N], base[BEST], ps[MT];
    __shared__ uint64_t head[MT / 64][64];
    __shared__ float top[BEST], pm[MT];
    __shared__ int count, passed, won[MT / 64], pass[MT], length[MT];
    __shared__ uint8_t taken[BEST * ((1 << 20) / BV)], over[BEST];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = blockIdx.x, W = a.n_beams, K = a.n_best;
    const int64_t row0 = (int64_t)g * W;
    const int L = W * nb;
    // the thread's first list, its part and its head (those of a finished beam's rows are not written, and not used), and the score of
    // the wave's first beam
    BeamPart p0 = {0.0, -INFINITY, 0};
    Cand c0 = {0.f, 0};
    if (tid < L) {
        p0 = parts[row0 * nb + tid];
        c0 = lists[(row0 * nb + tid) * K];
    }
    const float score = w < W ? a.scores[row0 + w] : 0.f;
    for (int b = tid; b < W; b += MT) over[b] = a.done != nullptr && a.done[row0 + b] ? 1 : 0;
    exp_table(tab);
    ps[tid] = p0.sum;
    pm[tid] = p0.max;
    if (tid == 0) count = passed = 0;
    __syncthreads();
    auto is_done = [&](int b) { return over[b] != 0; };
    // a row's sum: base + (z - m) is the score of a continuation (z - m first: of a row whose logits all are the type's
    // lowest value it is zero, and the sum's logarithm is not lost)
    for (int b = w; b < W; b += MT / 64) {
        const float sc = b == w ? score : a.scores[row0 + b];
        const bool done = is_done(b);
        float m = -INFINITY;
        double s = 0.0;
        if (!done) {
            auto part_max = [&](int j) { return b * nb + j < MT ? pm[b * nb + j] : parts[(row0 + b) * nb + j].max; };
            for (int j = lane; j < nb; j += 64) m = fmaxf(m, part_max(j));
            m = wave_max(m);
            if (m > -INFINITY)
                for (int j = lane; j < nb; j += 64)
                    s += (b * nb + j < MT ? ps[b * nb + j] : parts[(row0 + b) * nb + j].sum) * weight(part_max(j), m, 1.44269504088896340736, tab);
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
    auto entries = [&](int l) {
        const int b = l / nb;
        if (!(base[b] > -INFINITY)) return 0;
        if (is_done(b)) return l % nb == 0 ? 1 : 0;
        return l == tid ? p0.n : parts[row0 * nb + l].n;
    };
    auto make = [&](int l, const Cand& c, Entry& e) {
        const int b = l / nb;
        if (is_done(b)) {
            e = make_entry(base[b], b, 0.f, 0);
            return true;
        }
        if (top[b] == INFINITY && c.z < INFINITY) return false;       // infinite logits share the whole
        e = make_entry(base[b] + (top[b] == INFINITY ? 0.0 : (double)c.z - (double)top[b]), b, c.z, c.id);
        return true;
    };
    auto load = [&](int l, int r) { return is_done(l / nb) ? Cand{0.f, 0} : l == tid && r == 0 ? c0 : lists[(row0 * nb + l) * K + r]; };
    auto entry = [&](int l, int r, Entry& e) { return r < entries(l) && make(l, load(l, r), e); };
    auto emit = [&](int r, const Entry& e) {
        const int b = BEST - 1 - (int)(e.at >> 52);
        const bool was = is_done(b);
        const int id = was ? a.pad : 0xFFFFF - (int)(e.at & 0xFFFFF);
        const int64_t o = (int64_t)g * K + r;
        a.out_scores[o] = (float)unorder(e.score);
        a.out_parent[o] = b;
        a.out_ids[o] = id;
        if (a.out_done != nullptr) a.out_done[o] = was || id == a.eos;
    };
    // Of 64 groups of lists (a lane's, of all waves) the K-th largest of the groups' best heads is at most the K-th largest entry.
    // (Scores are kept as numbers in their order; none is 0.)
    uint64_t best = 0, first = 0;
    for (int l = tid; l < L; l += MT) {
        Entry e;
        if (entry(l, 0, e)) best = max(best, e.score);
        if (l == tid) first = best;
    }
    head[w][lane] = best;
    __syncthreads();
    best = head[0][lane];
#pragma unroll
    for (int j = 1; j < MT / 64; ++j) best = max(best, head[j][lane]);
    const uint64_t cut = max((uint64_t)kth_largest((uint32_t)(best >> 32), K, 8) << 32, (uint64_t)1);
    for (int l = tid; l < L; l += MT) {
        uint64_t s = first;
        if (l != tid) {
            Entry e;
            s = entry(l, 0, e) ? e.score : 0;
        }
        if (s >= cut) {
            const int i = atomicAdd(&passed, 1);
            if (i < MT) {
                pass[i] = l;
                length[i] = entries(l);
            }
        }
    }
    __syncthreads();
    for (int it = tid; it < min(passed, MT) * K; it += MT) {
        const int i = it / K, r = it % K;
        Entry e;
        if (r < length[i] && make(pass[i], load(pass[i], r), e) && e.score >= cut) {
            const int j = atomicAdd(&count, 1);
            if (j < ENT) ent[j] = e;
        }
    }
    __syncthreads();
    int n = count;
    if (n <= ENT && passed <= MT) {
        for (int i = tid; i < n; i += MT) {
            const int r = rank_of(ent, n, ent[i]);
            if (r < K) emit(r, ent[i]);
        }
    } else {
        // Many equal scores, or few long lists: the lists are merged head by head.
        for (int l = tid; l < L; l += MT) taken[l] = 0;
        Entry next;
        int from;
        auto heads = [&]() {               // the best head of the thread's lists
            from = -1;
            for (int l = tid; l < L; l += MT) {
                Entry e;
                if (taken[l] < K && entry(l, taken[l], e) && (from < 0 || next < e)) {
                    next = e;
                    from = l;
                }
            }
        };
        heads();
        for (n = 0; n < K; ++n) {
            Entry e = next;
            int l = from;
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) {
                const Entry y = {__shfl_xor(e.score, o, 64), __shfl_xor(e.at, o, 64)};
                const int yl = __shfl_xor(l, o, 64);
                if (yl >= 0 && (l < 0 || e < y)) {
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
                if (won[j] >= 0 && (l < 0 || e < ent[j])) {
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
    // a merge is bound by what one CU's waves issue, idle ones too (us for both kernels, with 256, 512 and 1024 threads: 128
    // entries 10.4, 10.7, 11.7; 1024 of 8 beams 13.5, 12.8, 13.8; 4096 35.9, 34.6, 35.0; 16384 34.4, 27.5, 26.6)
    const int entries = a.n_beams * nb * a.n_best;
    if (entries <= 512) FP_LAUNCH(merge_kernel<256>, dim3(a.n_groups), dim3(256), 0, st, a, nb, parts, lists);
    else if (entries <= 8192) FP_LAUNCH(merge_kernel<512>, dim3(a.n_groups), dim3(512), 0, st, a, nb, parts, lists);
    else FP_LAUNCH(merge_kernel<1024>, dim3(a.n_groups), dim3(1024), 0, st, a, nb, parts, lists);
    return hipGetLastError();
}

}  // namespace fpk
