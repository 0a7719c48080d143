// Sums and maxima of fp64 values over a wave (device code only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace nmm {

typedef unsigned wave_u32x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ double dpp_move(double x) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_mov_dpp(int(uint32_t(u)), CTRL, 0xF, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_mov_dpp(int(uint32_t(u >> 32)), CTRL, 0xF, 0xF, false);
    return __longlong_as_double((uint64_t(hi) << 32) | lo);
}

// x of the lanes 16 (32) apart: each pair of values in both lanes, in the same order.
__device__ __forceinline__ void row_pair16(double x, double* a, double* b) {
    const uint64_t u = __double_as_longlong(x);
    const wave_u32x2 lo = __builtin_amdgcn_permlane16_swap(uint32_t(u), uint32_t(u), false, false);
    const wave_u32x2 hi = __builtin_amdgcn_permlane16_swap(uint32_t(u >> 32), uint32_t(u >> 32), false, false);
    *a = __longlong_as_double((uint64_t(hi[0]) << 32) | lo[0]);
    *b = __longlong_as_double((uint64_t(hi[1]) << 32) | lo[1]);
}
__device__ __forceinline__ void row_pair32(double x, double* a, double* b) {
    const uint64_t u = __double_as_longlong(x);
    const wave_u32x2 lo = __builtin_amdgcn_permlane32_swap(uint32_t(u), uint32_t(u), false, false);
    const wave_u32x2 hi = __builtin_amdgcn_permlane32_swap(uint32_t(u >> 32), uint32_t(u >> 32), false, false);
    *a = __longlong_as_double((uint64_t(hi[0]) << 32) | lo[0]);
    *b = __longlong_as_double((uint64_t(hi[1]) << 32) | lo[1]);
}

// The sum over the wave in every lane, in a fixed order: quads, half rows, rows, then across rows.
__device__ __forceinline__ double sum64(double x) {
    x += dpp_move<0xB1>(x);
    x += dpp_move<0x4E>(x);
    x += dpp_move<0x141>(x);
    x += dpp_move<0x140>(x);
    double a, b;
    row_pair16(x, &a, &b);
    row_pair32(a + b, &a, &b);
    return a + b;
}

// The maximum over the wave in every lane; NaN counts as no value, and is the result where there is none.
__device__ __forceinline__ double max64(double x) {
    x = __builtin_fmax(x, dpp_move<0xB1>(x));
    x = __builtin_fmax(x, dpp_move<0x4E>(x));
    x = __builtin_fmax(x, dpp_move<0x141>(x));
    x = __builtin_fmax(x, dpp_move<0x140>(x));
    double a, b;
    row_pair16(x, &a, &b);
    row_pair32(__builtin_fmax(a, b), &a, &b);
    return __builtin_fmax(a, b);
}

}  // namespace nmm
