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
// exp(x) = 2^y, y = x log2 e = n / 256 + r, |r| <= 1 / 512: 2^(n / 256) from a table of 256 and the
// exponent, 2^r by its power series to the fourth order (the rest is below 4e-17).
//
// 32 sequences of 6 rows of 32000, T = 0.8: 9.3 us for the rows (24.6 MB; the exponentials' 64-bit arithmetic is some 6 of
// them), 10 for the masses and 8 for the draw, both chains of a dozen dependent loads.  One sequence of 4 rows, T = 0: 3.8 + 2.2.
#include <climits>

#include "fp_device.h"
#include "fp_internal.h"

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

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_d(double v) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, ROWS, 0xf, false),
                            __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, ROWS, 0xf, false));
}
// Inclusive sums over the wave's lanes.
__device__ __forceinline__ double wave_scan_d(double v) {
    v += dpp_d<0x111, 0xf>(v);
    v += dpp_d<0x112, 0xf>(v);
    v += dpp_d<0x114, 0xf>(v);
    v += dpp_d<0x118, 0xf>(v);
    v += dpp_d<0x142, 0xa>(v);
    v += dpp_d<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ double lane_d(double v, int l) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l));
}
__device__ __forceinline__ double wave_sum_d(double v) { return lane_d(wave_scan_d(v), 63); }

// 2^(n / 256), made by the compiler from the power series; a workgroup copies it to LDS (a barrier follows).
struct ExpTable {
    double v[256];
    constexpr ExpTable() : v() {
        for (int n = 0; n < 256; ++n) {
            const double x = n * 0.693147180559945309417 / 256.0;
            double s = 0.0;
            for (int k = 24; k >= 1; --k) s = (s + 1.0) * x / k;
            v[n] = 1.0 + s;
        }
    }
};
__device__ constexpr ExpTable EXP_TABLE;
__device__ __forceinline__ void exp_table(double* tab) { tab[threadIdx.x] = EXP_TABLE.v[threadIdx.x]; }
__device__ __forceinline__ double exp2_d(double y, const double* tab) {
    y = fmax(y, -1200.0);                  // 2^-1200 is zero
    constexpr double R = 6755399441055744.0 / 256.0;        // 1.5 2^52 / 256: adding it rounds to 1 / 256
    const double t = y + R;
    const int n = __double2loint(t);
    const double r = y - (t - R);
    constexpr double L = 0.693147180559945309417;
    double q = L * L * L * L / 24.0;
    q = fma(q, r, L * L * L / 6.0);
    q = fma(q, r, L * L / 2.0);
    q = fma(q, r, L);
    q = fma(q, r, 1.0);
    return ldexp(tab[n & 255] * q, n >> 8);
}
// exp((z - m) / T) with the weight rules: NaN and -inf have none, +inf all of it
__device__ __forceinline__ double weight(float z, float m, double c, const double* tab) {
    const double e = exp2_d(((double)z - (double)m) * c, tab);
    return z == m ? 1.0 : !(z > -INFINITY) || m == INFINITY ? 0.0 : e;
}

// The same for z that is no NaN and m < +inf, without the rules: -inf gives 2^-1200, zero, and m itself one.
__device__ __forceinline__ double weight_below(float z, double m, double c, const double* tab) {
    return exp2_d(((double)z - m) * c, tab);
}
__device__ __forceinline__ float no_nan(float z) { return fmaxf(z, -INFINITY); }

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
    __shared__ double sd[NT / 64], tab[NT];
    const int nb = gridDim.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t row = blockIdx.y;
    if (a.c > 0.0) exp_table(tab);
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
    if (a.c > 0.0 && m > -INFINITY) {
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
    __shared__ double tab[NT], sd[VB / CK][NT / 64];
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
    __shared__ double tab[NT], sd[NT / 64];
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

int blocks_of(int V) { return (V + VB - 1) / VB; }

}  // namespace

size_t verify_ws_bytes(int n_seqs, int n_rows, int V) {
    return (size_t)n_rows * blocks_of(V) * sizeof(Part) + (size_t)n_seqs * (blocks_of(V) * (VB / CK) * sizeof(double) + sizeof(Decision));
}

hipError_t launch_verify(const VerifyArgs& a, hipStream_t st) {
    const int nb = blocks_of(a.V);
    double* mass = (double*)((Part*)a.ws + (size_t)a.n_rows * nb);
    Decision* kept = (Decision*)(mass + (size_t)a.n_seqs * nb * (VB / CK));
    if (a.n_rows > 0) FP_LAUNCH(row_kernel, dim3(nb, a.n_rows), dim3(NT), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.c > 0.0) {
        FP_LAUNCH(mass_kernel, dim3(nb, a.n_seqs), dim3(NT), 0, st, a, mass, kept);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    FP_LAUNCH(pick_kernel, dim3(a.n_seqs), dim3(NT), 0, st, a, nb, mass, kept);
    return hipGetLastError();
}

}  // namespace fpk
