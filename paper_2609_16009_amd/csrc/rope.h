// RoPE angles, shared by the kernels that rotate (device code only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace nmm {

constexpr double kTwoPiHi = 6.283185307179586;          // 2*pi rounded to double
constexpr double kTwoPiLo = 2.4492935982947064e-16;     // 2*pi - kTwoPiHi
constexpr double kInvTwoPi = 0.15915494309189535;

// Sine and cosine of RoPE pair j's angle a = t * theta^(-2j/rope) = t * freq_step^j.  The power
// is taken by binary powering and a formed in fp64 (relative error a few units of 2^-53), then a
// is reduced to [-pi, pi] by a two-term Cody-Waite step with fused multiply-adds (k * kTwoPiHi
// is exact for |k| < 2^30, i.e. positions below 2^31); the sine and cosine of the reduced angle
// are taken in fp32.
__device__ __forceinline__ void rope_sincos(double freq_step, int64_t position, int j, float* sn, float* cs) {
    double f = 1.0, b = freq_step;
    for (int n = j; n; n >>= 1) {
        if (n & 1) f *= b;
        b *= b;
    }
    const double a = double(position) * f;
    const double k = rint(a * kInvTwoPi);
    const double r = fma(-k, kTwoPiLo, fma(-k, kTwoPiHi, a));
    sincosf(float(r), sn, cs);
}

}  // namespace nmm
