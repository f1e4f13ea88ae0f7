// Verification of drafted tokens against the target's logits, from given random numbers.
//
//     p_i = softmax(z_i / T);   x_i accepted if u_i q_i(x_i) < p_i(x_i);
//     at the first refusal one token from max(0, p_i - q_i), else one from the last row's p.
//
// Decisions are borders between floating-point numbers, so every sum and exponential that one
// depends on is in 64 bits: which order the sums take then changes a decision only where two
// numbers agree to some 1e-15.  Bound by reading the logits once (all rows: which one is refused
// is known only afterwards) and by the 64-bit exponentials, so the rows are spread over the whole
// GPU in blocks of VB ids:
//   row_kernel    per (row, block): maximum, its lowest id, sum of exp((z - max) / T)
//   mass_kernel   per (sequence, block): the accepted drafts are counted from the blocks' sums
//                 (every block's workgroup does so for itself), and the sums of the weights that the
//                 last token is drawn from, per CK ids
//   pick_kernel   per sequence: the CK ids that hold the draw, then the id; writes the tokens
// Greedy decoding (T = 0) needs the maxima only: row_kernel, pick_kernel.
//
// 32 sequences of 6 rows of 32000, T = 0.8: 9.3 us for the rows (24.6 MB; the exponentials' 64-bit arithmetic is some 6 of
// them), 10 for the masses and 8 for the draw, both chains of a dozen dependent loads.  One sequence of 4 rows, T = 0: 3.8 + 2.2.
#include "vocab.h"

namespace fpk {

namespace {

constexpr int VB = 4096;                   // ids per block
constexpr int CK = 1024;                   // ids per chunk of a draw: four per thread
constexpr int NT = 256;
constexpr int EPT = VB / NT;
static_assert(CK == 4 * NT && VB % CK == 0, "chunks");

struct Part {                              // one block of a row
    double sum;
    float max;
    int arg;
};

__device__ __forceinline__ int seq_row0(const VerifyArgs& a, int b) { return min(max(a.row_start[b], 0), a.n_rows); }
__device__ __forceinline__ int seq_rows(const VerifyArgs& a, int b) {
    return min(max(min(max(a.row_start[b + 1], 0), a.n_rows) - seq_row0(a, b), 0), a.max_rows);
}

// GREEDY: the maximum and its lowest id; else the maximum and the sum.
template <bool GREEDY>
__global__ void __launch_bounds__(NT, 8) row_kernel(VerifyArgs a) {
    __shared__ float sm[NT / 64];
    __shared__ int si[NT / 64];
    __shared__ double sd[NT / 64], tab[EXP_N];
    const int nb = gridDim.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.y;
    // past the row's end a load gives zeros
    const int v0 = blockIdx.x * VB, here = min(a.V - v0, VB);
    const auto z = buf_rsrc(a.logits + row * a.row_stride + v0, 4 * here);
    float x[EPT];
#pragma unroll
    for (int i = 0; i < EPT; ++i) x[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(z, 4 * tid, 4 * NT * i, 0));
    if (here < VB) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) x[i] = tid + NT * i < here ? x[i] : -INFINITY;
    }
    if (!GREEDY) exp_table(tab);
    float m = -INFINITY;
    int mi = INT_MAX;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
        if (!GREEDY) {
            m = fmaxf(m, x[i]);
        } else if (x[i] > m) {
            m = x[i];
            mi = v0 + tid + NT * i;
        }
    }
    if constexpr (GREEDY) {
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) {
            const float ov = __shfl_xor(m, o, 64);
            const int oi = __shfl_xor(mi, o, 64);
            best_of(m, mi, ov, oi);
        }
    } else {
        m = wave_max(m);
    }
    if (lane == 0) {
        sm[w] = m;
        si[w] = mi;
    }
    __syncthreads();
    m = sm[0];
    mi = si[0];
#pragma unroll
    for (int j = 1; j < NT / 64; ++j) best_of(m, mi, sm[j], si[j]);
    double s = 0.0;
    if (!GREEDY && m > -INFINITY) {
        if (m < INFINITY) {
            const double md = m;
#pragma unroll
            for (int i = 0; i < EPT; ++i) s += weight_below(no_nan(x[i]), md, a.c, tab);
        } else {
            int n = 0;
#pragma unroll
            for (int i = 0; i < EPT; ++i) n += x[i] == m ? 1 : 0;
            s = n;
        }
        s = wave_sum_d(s);
        if (lane == 0) sd[w] = s;
        __syncthreads();
        s = 0.0;
        for (int j = 0; j < NT / 64; ++j) s += sd[j];
    }
    if (tid == 0) ((Part*)a.ws)[row * nb + blockIdx.x] = Part{s, m, mi};
}

// What a sequence's rows decide: accepted drafts, and the deciding row's maximum, its id and sum.
struct Decision {
    double sum;
    int64_t row;
    int rows, acc, arg;
    float m;
};
__device__ __forceinline__ double draft_p(float q) { return q > 0.f ? (double)q : 0.0; }
// One wave; lane i judges draft i (max_rows is at most 64).
__device__ __forceinline__ Decision decide(const VerifyArgs& a, int nb, int b, const double* tab) {
    const int lane = threadIdx.x & 63;
    Decision d;
    d.rows = seq_rows(a, b);
    const int64_t r0 = seq_row0(a, b);
    const bool on = lane < d.rows, judge = lane < d.rows - 1;
    const int64_t row = r0 + lane;
    const Part* p = (const Part*)a.ws + row * nb;
    // the draft's own loads first: they lead to two more
    const int x = judge ? a.draft_ids[row] : -1;
    const bool in = x >= 0 && x < a.V;
    const float zx = in ? a.logits[row * a.row_stride + x] : -INFINITY;
    const float qx = in && a.draft_probs != nullptr ? a.draft_probs[row * a.draft_stride + x] : 1.f;
    const float ux = judge && a.c > 0.0 ? a.u[row] : 0.f;
    float m = -INFINITY;
    int mi = INT_MAX;
    double s = 0.0;
    bool ok = false;
    if (on) {
        // eight blocks' loads together, the running sum rescaled to the running maximum
        for (int j0 = 0; j0 < nb; j0 += 8) {
            Part q[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) q[j] = p[min(j0 + j, nb - 1)];
            const float old = m;
#pragma unroll
            for (int j = 0; j < 8; ++j) best_of(m, mi, q[j].max, q[j].arg);
            if (a.c > 0.0 && m > -INFINITY) {
                if (j0 > 0) s *= weight(old, m, a.c, tab);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j0 + j < nb) s += q[j].sum * weight(q[j].max, m, a.c, tab);
            }
        }
        if (in && m > -INFINITY) {
            if (a.c > 0.0) ok = (double)ux * draft_p(qx) * s < weight(zx, m, a.c, tab);
            else ok = x == mi;
        }
    }
    d.acc = __builtin_ctzll(~__ballot(ok));           // lanes from rows - 1 on never accept
    d.row = r0 + d.acc;
    d.m = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(m), d.acc));
    d.arg = __builtin_amdgcn_readlane(mi, d.acc);
    d.sum = lane_d(s, d.acc);
    return d;
}

// Weights of four ids from v on in the last draw: p - q (not below zero) at a refused draft, p at the
// last row, and p at a refused draft too when `plain` (p - q is zero everywhere).
__device__ __forceinline__ void draw_weights(const VerifyArgs& a, const Decision& d, int v, bool plain, const double* tab,
                                             double (&wt)[4]) {
    const float* z = a.logits + d.row * a.row_stride;
    const bool whole = plain || d.acc == d.rows - 1, qs = !whole && a.draft_probs != nullptr;
    const float* q = a.draft_probs + d.row * a.draft_stride;
    const int x = !whole && !qs ? a.draft_ids[d.row] : -1;
    const double inv = 1.0 / d.sum;
    float zz[4], qq[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool in = v + i < a.V;
        zz[i] = in ? z[v + i] : -INFINITY;
        qq[i] = in && qs ? q[v + i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double p = (d.m < INFINITY ? weight_below(no_nan(zz[i]), d.m, a.c, tab) : zz[i] == d.m ? 1.0 : 0.0) * inv;
        wt[i] = v + i == x ? 0.0 : fmax(p - draft_p(qq[i]), 0.0);
    }
}

__global__ void __launch_bounds__(NT) mass_kernel(VerifyArgs a, double* __restrict__ mass, Decision* __restrict__ kept) {
    __shared__ double tab[EXP_N], sd[VB / CK][NT / 64];
    const int nb = gridDim.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    exp_table(tab);
    __syncthreads();
    const Decision d = decide(a, nb, b, tab);
    if (blockIdx.x == 0 && tid == 0) kept[b] = d;
    const bool live = d.rows > 0 && d.m > -INFINITY;
#pragma unroll
    for (int c = 0; c < VB / CK; ++c) {
        double wt[4] = {0.0, 0.0, 0.0, 0.0};
        if (live) draw_weights(a, d, blockIdx.x * VB + c * CK + 4 * tid, false, tab, wt);
        const double s = wave_sum_d((wt[0] + wt[1]) + (wt[2] + wt[3]));
        if (lane == 0) sd[c][w] = s;
    }
    __syncthreads();
    if (tid < VB / CK) mass[((int64_t)b * nb + blockIdx.x) * (VB / CK) + tid] = (sd[tid][0] + sd[tid][1]) + (sd[tid][2] + sd[tid][3]);
}

// One workgroup per sequence.  The chunk that holds the draw from the chunks' masses, then the id in it.
__global__ void __launch_bounds__(NT) pick_kernel(VerifyArgs a, int nb, const double* __restrict__ mass, const Decision* __restrict__ kept) {
    __shared__ double tab[EXP_N], sd[NT / 64];
    __shared__ int found, top;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    exp_table(tab);
    if (tid == 0) {
        found = INT_MAX;
        top = -1;
    }
    __syncthreads();
    const Decision d = a.c > 0.0 ? kept[b] : decide(a, nb, b, tab);
    int last = -1;
    if (d.rows > 0 && d.m > -INFINITY) {
        if (a.c == 0.0) {
            last = d.arg;
        } else {
            // sum of chunk j of the draw: of p - q, or of p where that is zero everywhere (the chunks of p
            // are then taken as whole blocks, of their first chunk)
            const double* ms = mass + (int64_t)b * nb * (VB / CK);
            const Part* pp = (const Part*)a.ws + d.row * nb;
            const int nc = nb * (VB / CK);
            bool plain = false;
            auto chunk_mass = [&](int j) {
                if (j >= nc) return 0.0;
                if (!plain) return ms[j];
                const Part& p = pp[j / (VB / CK)];
                return j % (VB / CK) ? 0.0 : p.sum * weight(p.max, d.m, a.c, tab) / d.sum;
            };
            double total = 0.0;
            for (int j0 = 0; j0 < nc; j0 += 64) total += wave_sum_d(chunk_mass(j0 + lane));
            if (!(total > 0.0)) {
                plain = true;
                total = 0.0;
                for (int j0 = 0; j0 < nc; j0 += 64) total += wave_sum_d(chunk_mass(j0 + lane));
            }
            const double goal = (double)a.u_last[b] * total;
            // the first chunk whose running sum passes the goal; rounding may leave the goal at the
            // total: then the last chunk with any mass, and in it the last id with any
            double base = 0.0, at = 0.0;
            int ck = -1;
            for (int j0 = 0; j0 < nc; j0 += 64) {
                const double mj = chunk_mass(j0 + lane), inc = base + wave_scan_d(mj);
                const uint64_t any = __ballot(mj > 0.0), past = any & __ballot(inc > goal);
                if (any) {
                    const int l = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
                    ck = j0 + l;
                    at = lane_d(inc - mj, l);
                    if (past) break;
                }
                base = lane_d(inc, 63);
            }
            const int chunks = plain ? VB / CK : 1;
            for (int c = 0; c < chunks && ck >= 0; ++c) {
                double wt[4];
                const int v0 = (ck + c) * CK + 4 * tid;
                draw_weights(a, d, v0, plain, tab, wt);
                const double s = (wt[0] + wt[1]) + (wt[2] + wt[3]);
                const double inc = wave_scan_d(s);
                if (lane == 63) sd[w] = inc;
                __syncthreads();
                double run = at + (inc - s), chunk = 0.0;
                for (int j = 0; j < NT / 64; ++j) {
                    if (j < w) run += sd[j];
                    chunk += sd[j];
                }
                int hi = -1;
#pragma unroll
                for (int i = 3; i >= 0; --i)
                    if (wt[i] > 0.0 && hi < 0) hi = v0 + i;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    run += wt[i];
                    if (wt[i] > 0.0 && run > goal) {
                        atomicMin(&found, v0 + i);
                        break;
                    }
                }
                if (hi >= 0) atomicMax(&top, hi);
                at += chunk;
                __syncthreads();
                if (found != INT_MAX) break;
            }
            last = found != INT_MAX ? found : top;
        }
    }
    for (int i = tid; i < a.max_rows; i += NT)
        a.out_ids[(int64_t)b * a.max_rows + i] = i < d.acc ? a.draft_ids[d.row - d.acc + i] : i == d.acc && d.rows > 0 ? last : -1;
    if (tid == 0) a.n_out[b] = d.rows > 0 ? d.acc + 1 : 0;
}

// ---- trees
//
// A tree's decision is that of one draw: with y_i drawn from p_i, node by node from the root on, the child that holds
// y_i is accepted and a node without such a child ends the path with y_i.  Whatever the tree is, the tokens are those
// that the target alone would draw.  Every node's draw is independent of the path, so all are made at once and only the
// walk remains:
//   row_kernel    as above
//   draw_kernel   per row: the block that holds the draw by the blocks' sums, then the id in it
//   walk_kernel   per sequence, one wave, lane i its node i (T = 0: a node's token is its row's maximum)
//
// 16 trees of up to 48 nodes (383 rows) over 32000 ids, T = 0.8: 15 us for the rows (49 MB, 3.2 TB/s), 7 for the draws, each a chain of
// the blocks' sums, the ids of one block and two joins over its waves, and 2.5 for the walks.  One tree of 8 nodes, T = 0: 3.9 + 2.5.

constexpr int DT = 1024, DPT = VB / DT;     // threads of a draw, ids of one
__global__ void __launch_bounds__(DT) draw_kernel(VerifyArgs a, int nb, int* __restrict__ drawn) {
    __shared__ double tab[EXP_N], sd[2][DT / 64], before;
    __shared__ float sm[DT / 64];
    __shared__ int first[2], last[2];
    static_assert(DT >= (1 << 20) / VB, "a thread per block of the largest vocabulary");
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.x;
    const Part p = tid < nb ? ((const Part*)a.ws)[row * nb + tid] : Part{0.0, -INFINITY, INT_MAX};
    exp_table(tab);
    if (tid < 2) {
        first[tid] = INT_MAX;
        last[tid] = -1;
    }
    float m = wave_max(p.max);
    if (lane == 0) sm[w] = m;
    __syncthreads();
    const int waves = (nb + 63) / 64;
    m = sm[0];
    for (int j = 1; j < waves; ++j) m = fmaxf(m, sm[j]);
    if (!(m > -INFINITY)) {
        if (tid == 0) drawn[row] = -1;
        return;
    }
    // the first block whose running sum passes the goal; rounding may leave the goal at the total: then the
    // last block with any mass, and in it the last id with any
    double mass = 0.0, inc = 0.0, total = 0.0;
    if (w < waves) {
        mass = tid < nb ? p.sum * weight(p.max, m, a.c, tab) : 0.0;
        inc = wave_scan_d(mass);
        if (lane == 63) sd[0][w] = inc;
    }
    __syncthreads();
    for (int j = 0; j < waves; ++j) {
        if (j == w) inc += total;
        total += sd[0][j];
    }
    const double goal = (double)a.u[row] * total;
    if (mass > 0.0) {
        if (inc > goal) atomicMin(&first[0], tid);
        atomicMax(&last[0], tid);
    }
    __syncthreads();
    const int blk = first[0] != INT_MAX ? first[0] : last[0];
    if (tid == blk) before = inc - mass;
    // DPT ids in a row per thread
    const int at0 = blk * VB, v0 = at0 + DPT * tid, here = min(a.V - at0, VB);
    const auto z = buf_rsrc(a.logits + row * a.row_stride + at0, 4 * here);
    float x[DPT];
    double wt[DPT], s = 0.0;
#pragma unroll
    for (int i = 0; i < DPT; ++i) x[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(z, 4 * (DPT * tid + i), 0, 0));
#pragma unroll
    for (int i = 0; i < DPT; ++i) {
        wt[i] = DPT * tid + i < here ? weight(x[i], m, a.c, tab) : 0.0;
        s += wt[i];
    }
    inc = wave_scan_d(s);
    if (lane == 63) sd[1][w] = inc;
    __syncthreads();
    double run = before + (inc - s);
    for (int j = 0; j < w; ++j) run += sd[1][j];
    int at = INT_MAX, hi = -1;
#pragma unroll
    for (int i = 0; i < DPT; ++i) {
        run += wt[i];
        if (wt[i] > 0.0) {
            hi = v0 + i;
            if (run > goal) at = min(at, v0 + i);
        }
    }
    // one lane of a wave has the wave's lowest, one its highest
    const uint64_t past = __ballot(at != INT_MAX), any = __ballot(hi >= 0);
    if (past != 0 && lane == __builtin_ctzll(past)) atomicMin(&first[1], at);
    if (any != 0 && lane == 63 - __builtin_clzll(any)) atomicMax(&last[1], hi);
    __syncthreads();
    if (tid == 0) drawn[row] = first[1] != INT_MAX ? first[1] : last[1];
}

__global__ void __launch_bounds__(64) walk_kernel(VerifyArgs a, int nb, const int* __restrict__ drawn, const int* __restrict__ parent,
                                                  int* __restrict__ path) {
    const int b = blockIdx.x, lane = threadIdx.x, n = seq_rows(a, b);
    const int64_t row = seq_row0(a, b) + lane;
    int p = -1, id = -1, y = -1;
    if (lane < n) {
        p = parent[row];
        id = a.draft_ids[row];
        if (p >= lane) p = -1;
        if (a.c > 0.0) {
            y = drawn[row];
        } else {
            const Part* q = (const Part*)a.ws + row * nb;
            float m = -INFINITY;
            int mi = INT_MAX;
            for (int j0 = 0; j0 < nb; j0 += 8) {
                Part x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = q[min(j0 + j, nb - 1)];
#pragma unroll
                for (int j = 0; j < 8; ++j) best_of(m, mi, x[j].max, x[j].arg);
            }
            y = m > -INFINITY ? mi : -1;
        }
    }
    int at = 0, k = 0, tok = -1, node = -1;
    while (k < n) {
        const int yc = __builtin_amdgcn_readlane(y, at);
        if (lane == k) {
            tok = yc;
            node = at;
        }
        ++k;
        const uint64_t hit = __ballot(p == at && id == yc && yc >= 0);
        if (hit == 0) break;
        at = __builtin_ctzll(hit);
    }
    if (lane < a.max_rows) {
        a.out_ids[(int64_t)b * a.max_rows + lane] = tok;
        path[(int64_t)b * a.max_rows + lane] = node;
    }
    if (lane == 0) a.n_out[b] = k;
}

int blocks_of(int V) { return (V + VB - 1) / VB; }

hipError_t launch_rows(const VerifyArgs& a, int nb, hipStream_t st) {
    if (a.n_rows > 0 && a.c > 0.0) FP_LAUNCH(row_kernel<false>, dim3(nb, a.n_rows), dim3(NT), 0, st, a);
    else if (a.n_rows > 0) FP_LAUNCH(row_kernel<true>, dim3(nb, a.n_rows), dim3(NT), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t verify_tree_ws_bytes(int n_rows, int V) { return (size_t)n_rows * (blocks_of(V) * sizeof(Part) + sizeof(int)); }

hipError_t launch_verify_tree(const VerifyArgs& a, const int* parent, int* path, hipStream_t st) {
    const int nb = blocks_of(a.V);
    int* drawn = (int*)((Part*)a.ws + (size_t)a.n_rows * nb);
    hipError_t e = launch_rows(a, nb, st);
    if (e != hipSuccess) return e;
    if (a.c > 0.0 && a.n_rows > 0) {
        FP_LAUNCH(draw_kernel, dim3(a.n_rows), dim3(DT), 0, st, a, nb, drawn);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    FP_LAUNCH(walk_kernel, dim3(a.n_seqs), dim3(64), 0, st, a, nb, drawn, parent, path);
    return hipGetLastError();
}

size_t verify_ws_bytes(int n_seqs, int n_rows, int V) {
    return (size_t)n_rows * blocks_of(V) * sizeof(Part) + (size_t)n_seqs * (blocks_of(V) * (VB / CK) * sizeof(double) + sizeof(Decision));
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
    const int nb = blocks_of(a.V);
    double* mass = (double*)((Part*)a.ws + (size_t)a.n_rows * nb);
    Decision* kept = (Decision*)(mass + (size_t)a.n_seqs * nb * (VB / CK));
    hipError_t e = launch_rows(a, nb, st);
    if (e != hipSuccess) return e;
    if (a.c > 0.0) {
        FP_LAUNCH(mass_kernel, dim3(nb, a.n_seqs), dim3(NT), 0, st, a, mass, kept);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    FP_LAUNCH(pick_kernel, dim3(a.n_seqs), dim3(NT), 0, st, a, nb, mass, kept);
    return hipGetLastError();
}

}  // namespace fpk
