// RoPE angles, shared by the kernels that rotate (device code only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace nmm {

constexpr double kTwoPiHi = 6.283185307179586;          // 2*pi rounded to double
constexpr double kTwoPiLo = 2.4492935982947064e-16;     // 2*pi - kTwoPiHi
constexpr double kInvTwoPi = 0.15915494309189535;

// RoPE pair j's angle a = t * theta^(-2j/rope) = t * freq_step^j, reduced to [-pi, pi].  The power
// is taken by binary powering and a formed in fp64 (relative error a few units of 2^-53), then a
// is reduced by a two-term Cody-Waite step with fused multiply-adds (k * kTwoPiHi
// is exact for |k| < 2^30, i.e. positions below 2^31).
__device__ __forceinline__ double rope_reduced(double freq_step, int64_t position, int j) {
    double f = 1.0, b = freq_step;
    for (int n = j; n; n >>= 1) {
        if (n & 1) f *= b;
        b *= b;
    }
    const double a = double(position) * f;
    const double k = rint(a * kInvTwoPi);
    return fma(-k, kTwoPiLo, fma(-k, kTwoPiHi, a));
}

// The angle's sine and cosine in fp32.
__device__ __forceinline__ void rope_sincos(double freq_step, int64_t position, int j, float* sn, float* cs) {
    sincosf(float(rope_reduced(freq_step, position, j)), sn, cs);
}

// The same in fp64, to about 2e-14 (the angle's own error aside): Taylor's series about the nearest multiple of pi / 2, to
// t^13 and t^14.
__device__ __forceinline__ void rope_sincos64(double freq_step, int64_t position, int j, double* sn, double* cs) {
    const double r = rope_reduced(freq_step, position, j);
    const double q = rint(r * (4 * kInvTwoPi));
    const double t = fma(-q, kTwoPiLo / 4, fma(-q, kTwoPiHi / 4, r)), u = t * t;
    double s = fma(u, 1.0 / 6227020800.0, -1.0 / 39916800.0), c = fma(u, -1.0 / 87178291200.0, 1.0 / 479001600.0);
    s = fma(u, s, 1.0 / 362880.0);
    c = fma(u, c, -1.0 / 3628800.0);
    s = fma(u, s, -1.0 / 5040.0);
    c = fma(u, c, 1.0 / 40320.0);
    s = fma(u, s, 1.0 / 120.0);
    c = fma(u, c, -1.0 / 720.0);
    s = fma(u, s, -1.0 / 6.0);
    c = fma(u, c, 1.0 / 24.0);
    s = fma(u * t, s, t);
    c = fma(u, c, -0.5);
    c = fma(u, c, 1.0);
    const int n = int(q) & 3;                       // sin(t + n pi / 2) and cos
    const double x = n & 1 ? c : s, y = n & 1 ? s : c;
    *sn = n & 2 ? -x : x;
    *cs = (n + 1) & 2 ? -y : y;
}

}  // namespace nmm
