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
//                 (every block's workgroup does so for itself), and the sum of the weights that
//                 the last token is drawn from
//   pick_kernel   per sequence: the block that holds the draw, then the id in it; writes the tokens
// Greedy decoding (T = 0) needs the maxima only: row_kernel, pick_kernel.
#include <climits>

#include "fp_device.h"
#include "fp_internal.h"

namespace fpk {

namespace {

constexpr int VB = 4096;                   // ids per block
constexpr int NT = 256;
constexpr int EPT = VB / NT;

struct Part {                              // one block of a row
    double sum;
    float max;
    int arg;
};

__device__ __forceinline__ double shfl_xor_d(double v, int o) {
    return __hiloint2double(__shfl_xor(__double2hiint(v), o, 64), __shfl_xor(__double2loint(v), o, 64));
}
__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += shfl_xor_d(v, o);
    return v;
}

// exp((z - m) / T) with the weight rules: NaN and -inf have none, +inf all of it
__device__ __forceinline__ double weight(float z, float m, double inv_t) {
    if (z == m) return 1.0;
    if (!(z > -INFINITY) || m == INFINITY) return 0.0;
    return exp(((double)z - (double)m) * inv_t);
}

// the larger value, the lower id among equal ones
__device__ __forceinline__ void best_of(float& v, int& i, float ov, int oi) {
    if (ov > v || (ov == v && oi < i)) {
        v = ov;
        i = oi;
    }
}

__device__ __forceinline__ int seq_row0(const VerifyArgs& a, int b) { return min(max(a.row_start[b], 0), a.n_rows); }
__device__ __forceinline__ int seq_rows(const VerifyArgs& a, int b) {
    return min(max(min(max(a.row_start[b + 1], 0), a.n_rows) - seq_row0(a, b), 0), a.max_rows);
}

__global__ void __launch_bounds__(NT) row_kernel(VerifyArgs a) {
    __shared__ float sm[NT / 64];
    __shared__ int si[NT / 64];
    __shared__ double sd[NT / 64];
    const int nb = gridDim.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.y;
    const int v0 = blockIdx.x * VB;
    const float* z = a.logits + row * a.row_stride;
    float x[EPT];
    float m = -INFINITY;
    int mi = INT_MAX;
#pragma unroll
    for (int i = 0; i < EPT; ++i) {
        const int v = v0 + tid + NT * i;
        x[i] = v < a.V ? z[v] : -INFINITY;
        if (x[i] > m) {
            m = x[i];
            mi = v;
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const float ov = __shfl_xor(m, o, 64);
        const int oi = __shfl_xor(mi, o, 64);
        best_of(m, mi, ov, oi);
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
    if (a.inv_t > 0.0 && m > -INFINITY) {
#pragma unroll
        for (int i = 0; i < EPT; ++i) s += weight(x[i], m, a.inv_t);
        s = wave_sum_d(s);
        if (lane == 0) sd[w] = s;
        __syncthreads();
        s = 0.0;
        for (int j = 0; j < NT / 64; ++j) s += sd[j];
    }
    if (tid == 0) ((Part*)a.ws)[row * nb + blockIdx.x] = Part{s, m, mi};
}

// The row's maximum, its lowest id and the sum of its weights (one lane's own row).
__device__ __forceinline__ void row_total(const VerifyArgs& a, int nb, int64_t row, float& m, int& mi, double& s) {
    const Part* p = (const Part*)a.ws + row * nb;
    m = -INFINITY;
    mi = INT_MAX;
    for (int j = 0; j < nb; ++j) best_of(m, mi, p[j].max, p[j].arg);
    s = 0.0;
    if (a.inv_t > 0.0)
        for (int j = 0; j < nb; ++j)
            if (p[j].max > -INFINITY) s += p[j].sum * weight(p[j].max, m, a.inv_t);
}

// What a sequence's rows decide: accepted drafts, and the deciding row's maximum and sum.
struct Decision {
    int rows, acc;
    int64_t row;
    float m;
    int arg;
    double sum;
};
__device__ __forceinline__ double draft_p(const VerifyArgs& a, int64_t row, int x) {
    if (a.draft_probs == nullptr) return 1.0;
    const double q = (double)a.draft_probs[row * a.draft_stride + x];
    return q > 0.0 ? q : 0.0;
}
// One wave; lane i judges draft i (max_rows is at most 64).
__device__ __forceinline__ Decision decide(const VerifyArgs& a, int nb, int b) {
    const int lane = threadIdx.x & 63;
    Decision d;
    d.rows = seq_rows(a, b);
    const int64_t r0 = seq_row0(a, b);
    float m = -INFINITY;
    int mi = INT_MAX;
    double s = 0.0;
    bool ok = false;
    if (lane < d.rows) {
        const int64_t row = r0 + lane;
        row_total(a, nb, row, m, mi, s);
        if (lane < d.rows - 1) {
            const int x = a.draft_ids[row];
            if (x >= 0 && x < a.V && m > -INFINITY) {
                if (a.inv_t > 0.0) {
                    const double p = weight(a.logits[row * a.row_stride + x], m, a.inv_t) / s;
                    ok = (double)a.u[row] * draft_p(a, row, x) < p;
                } else {
                    ok = x == mi;
                }
            }
        }
    }
    d.acc = __builtin_ctzll(~__ballot(ok));           // lanes from rows - 1 on never accept
    d.row = r0 + d.acc;
    d.m = __shfl(m, d.acc, 64);
    d.arg = __shfl(mi, d.acc, 64);
    d.sum = __hiloint2double(__shfl(__double2hiint(s), d.acc, 64), __shfl(__double2loint(s), d.acc, 64));
    return d;
}

// Weight of id v in the last draw: p - q (not below zero) at a refused draft, p at the last row,
// and p at a refused draft too when `plain` (p - q is zero everywhere).
__device__ __forceinline__ double draw_weight(const VerifyArgs& a, const Decision& d, int v, bool plain) {
    const double p = weight(a.logits[d.row * a.row_stride + v], d.m, a.inv_t) / d.sum;
    if (plain || d.acc == d.rows - 1) return p;
    if (a.draft_probs == nullptr) return v == a.draft_ids[d.row] ? 0.0 : p;
    return fmax(p - draft_p(a, d.row, v), 0.0);
}

__global__ void __launch_bounds__(NT) mass_kernel(VerifyArgs a, double* __restrict__ mass) {
    __shared__ double sd[2][NT / 64];
    const int nb = gridDim.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const Decision d = decide(a, nb, b);
    double s = 0.0, sp = 0.0;
    if (d.rows > 0 && d.m > -INFINITY) {
        const int v0 = blockIdx.x * VB;
        for (int i = 0; i < EPT; ++i) {
            const int v = v0 + tid + NT * i;
            if (v < a.V) {
                s += draw_weight(a, d, v, false);
                sp += draw_weight(a, d, v, true);
            }
        }
    }
    s = wave_sum_d(s);
    sp = wave_sum_d(sp);
    if (lane == 0) {
        sd[0][w] = s;
        sd[1][w] = sp;
    }
    __syncthreads();
    if (tid < 2) {
        double t = 0.0;
        for (int j = 0; j < NT / 64; ++j) t += sd[tid][j];
        mass[((int64_t)b * nb + blockIdx.x) * 2 + tid] = t;
    }
}

// One workgroup per sequence.  The draw's block from the blocks' masses, then 1024 ids at a time
// in id order: four per lane, prefix sums over the workgroup.
__global__ void __launch_bounds__(NT) pick_kernel(VerifyArgs a, int nb, const double* __restrict__ mass) {
    __shared__ double sd[NT / 64];
    __shared__ int found, top;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const Decision d = decide(a, nb, b);
    int last = -1;
    if (d.rows > 0 && d.m > -INFINITY) {
        if (a.inv_t == 0.0) {
            last = d.arg;
        } else {
            const double* ms = mass + (int64_t)b * nb * 2;
            double total = 0.0;
            for (int j = 0; j < nb; ++j) total += ms[2 * j];
            const bool plain = !(total > 0.0);
            if (plain) {
                total = 0.0;
                for (int j = 0; j < nb; ++j) total += ms[2 * j + 1];
            }
            const double goal = (double)a.u_last[b] * total;
            // the first block whose running sum passes the goal; rounding may leave the goal at the
            // total: then the last block with any mass, and in it the last id with any
            double base = 0.0;
            int blk = -1;
            double at = 0.0;
            for (int j = 0; j < nb; ++j) {
                const double mj = ms[2 * j + plain];
                if (mj > 0.0) {
                    blk = j;
                    at = base;
                    if (base + mj > goal) break;
                }
                base += mj;
            }
            if (tid == 0) {
                found = INT_MAX;
                top = -1;
            }
            __syncthreads();
            for (int c = 0; c < VB && blk >= 0; c += 4 * NT) {
                double wt[4], s = 0.0;
                int hi = -1;
                const int v0 = blk * VB + c + 4 * tid;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    wt[i] = v0 + i < a.V ? draw_weight(a, d, v0 + i, plain) : 0.0;
                    if (wt[i] > 0.0) hi = v0 + i;
                    s += wt[i];
                }
                double inc = s;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const double t = __hiloint2double(__shfl_up(__double2hiint(inc), o, 64), __shfl_up(__double2loint(inc), o, 64));
                    if (lane >= o) inc += t;
                }
                if (lane == 63) sd[w] = inc;
                __syncthreads();
                double run = at + (inc - s), chunk = 0.0;
                for (int j = 0; j < NT / 64; ++j) {
                    if (j < w) run += sd[j];
                    chunk += sd[j];
                }
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

int blocks_of(int V) { return (V + VB - 1) / VB; }

}  // namespace

size_t verify_ws_bytes(int n_seqs, int n_rows, int V) {
    return (size_t)n_rows * blocks_of(V) * sizeof(Part) + (size_t)n_seqs * blocks_of(V) * 2 * sizeof(double);
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
    const int nb = blocks_of(a.V);
    double* mass = (double*)((Part*)a.ws + (size_t)a.n_rows * nb);
    if (a.n_rows > 0) FP_LAUNCH(row_kernel, dim3(nb, a.n_rows), dim3(NT), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.inv_t > 0.0) {
        FP_LAUNCH(mass_kernel, dim3(nb, a.n_seqs), dim3(NT), 0, st, a, mass);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    FP_LAUNCH(pick_kernel, dim3(a.n_seqs), dim3(NT), 0, st, a, nb, mass);
    return hipGetLastError();
}

}  // namespace fpk
