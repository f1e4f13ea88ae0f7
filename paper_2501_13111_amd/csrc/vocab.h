// Sums over a row of logits in 64 bits, for decisions that are borders between such sums: exponentials from a
// table, sums over a wave, and the weight of a logit with its rules.
//
// exp(x) = 2^y, y = x log2 e = n / N + r, |r| <= 1 / (2 N): 2^(n / N) from a table of N and the exponent, 2^r by its
// power series.  N = 256 with the fourth order leaves less than 4e-17, N = 32 with the fifth 2.3e-15, what the roundings
// of a sum of thousands may leave too (24 groups of 8 beams over 128000 ids: 32.2 us; with the fourth, 1.3e-12, 31.9; with the sixth 32.9).
#pragma once
#include <climits>

#include "fp_device.h"
#include "fp_internal.h"

namespace fpk {

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

// 2^(n / N), made by the compiler from the power series; a workgroup copies it to LDS (a barrier follows).
template <int N>
struct ExpTable {
    double v[N];
    constexpr ExpTable() : v() {
        for (int n = 0; n < N; ++n) {
            const double x = n * 0.693147180559945309417 / N;
            double s = 0.0;
            for (int k = 24; k >= 1; --k) s = (s + 1.0) * x / k;
            v[n] = 1.0 + s;
        }
    }
};
template <int N>
__device__ constexpr ExpTable<N> EXP_TABLE;
template <int N>
__device__ __forceinline__ void exp_table(double (&tab)[N]) {
    if (threadIdx.x < N) tab[threadIdx.x] = EXP_TABLE<N>.v[threadIdx.x];
}
constexpr int EXP_N = 256;
// 2^y for y >= -1022 or so
template <int N>
__device__ __forceinline__ double exp2_series(double y, const double* tab) {
    constexpr double R = 6755399441055744.0 / N;            // 1.5 2^52 / N: adding it rounds to 1 / N
    const double t = y + R;
    const int n = __double2loint(t);
    const double r = y - (t - R);
    constexpr double L = 0.693147180559945309417;
    double q = L * L * L * L / 24.0;
    if constexpr (N < 256) q = fma(L * L * L * L * L / 120.0, r, q);
    q = fma(q, r, L * L * L / 6.0);
    q = fma(q, r, L * L / 2.0);
    q = fma(q, r, L);
    q = fma(q, r, 1.0);
    return ldexp(tab[n & (N - 1)] * q, n >> (N == 256 ? 8 : 5));
}
__device__ __forceinline__ double exp2_d(double y, const double* tab) { return exp2_series<EXP_N>(fmax(y, -1200.0), tab); }        // 2^-1200 is zero
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

}  // namespace fpk
