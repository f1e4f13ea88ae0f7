// Sums over a row of logits in 64 bits, for decisions that are borders between such sums: exponentials from a
// table, sums over a wave, and the weight of a logit with its rules.
//
// exp(x) = 2^y, y = x log2 e = n / 32 + r, |r| <= 1 / 64: 2^(n / 32) from a table of 32 and the exponent, 2^r by its
// power series to the sixth order (the rest is below 4e-18).  A table of 256 with the fourth order takes two operations less,
// but its entries share the banks of LDS, and a wave's lookups wait for each other.
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

// 2^(n / 32), made by the compiler from the power series; a workgroup copies it to LDS (a barrier follows).
constexpr int EXP_N = 32;
struct ExpTable {
    double v[EXP_N];
    constexpr ExpTable() : v() {
        for (int n = 0; n < EXP_N; ++n) {
            const double x = n * 0.693147180559945309417 / EXP_N;
            double s = 0.0;
            for (int k = 24; k >= 1; --k) s = (s + 1.0) * x / k;
            v[n] = 1.0 + s;
        }
    }
};
__device__ constexpr ExpTable EXP_TABLE;
__device__ __forceinline__ void exp_table(double* tab) {
    if (threadIdx.x < EXP_N) tab[threadIdx.x] = EXP_TABLE.v[threadIdx.x];
}
// 2^y for y >= -1022 with ORDER terms of the series
template <int ORDER>
__device__ __forceinline__ double exp2_series(double y, const double* tab) {
    constexpr double R = 6755399441055744.0 / EXP_N;        // 1.5 2^52 / 32: adding it rounds to 1 / 32
    constexpr double L = 0.693147180559945309417, C[] = {1.0, L, L * L / 2.0, L * L * L / 6.0, L * L * L * L / 24.0, L * L * L * L * L / 120.0,
                                                         L * L * L * L * L * L / 720.0};
    const double t = y + R;
    const int n = __double2loint(t);
    const double r = y - (t - R);
    double q = C[ORDER];
#pragma unroll
    for (int k = ORDER - 1; k >= 0; --k) q = fma(q, r, C[k]);
    return ldexp(tab[n & (EXP_N - 1)] * q, n >> 5);
}
__device__ __forceinline__ double exp2_d(double y, const double* tab) { return exp2_series<6>(fmax(y, -1200.0), tab); }        // 2^-1200 is zero
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
