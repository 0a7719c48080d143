// Conversions to bf16 shared by the kernels (device code only).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace nmm {

// Nearest, ties to even (the hardware conversion).
__device__ __forceinline__ uint16_t to_bf16_bits(float v) {
    return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
}

// Nearest, ties away from zero: adding half of the dropped range to the magnitude bits carries
// into the kept bits exactly when the dropped part is at least one half (a carry out of the
// largest finite value ends at infinity, as it should).  NaN stays a quiet NaN.
__device__ __forceinline__ uint16_t to_bf16_bits_away(float v) {
    const uint32_t u = __float_as_uint(v);
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return static_cast<uint16_t>((u >> 16) | 0x40u);
    return static_cast<uint16_t>((u + 0x8000u) >> 16);
}

__device__ __forceinline__ uint16_t to_bf16_mode(float v, int away) {
    return away ? to_bf16_bits_away(v) : to_bf16_bits(v);
}

// A double as a float on its way to bf16: its first 21 bits, the last of them set where later ones were ("to odd"), so that the
// float lies on a boundary between two bf16 numbers only where the double does and rounding it is rounding the double once.  (A
// nearest float may be such a boundary, from which the value then goes to even: 9 of 10^6 of RMSNorm's and RoPE's values.)
// Below 2^-126, among the subnormals, the conversion to float may still round.  8192 cache rows written and read 14.5 us with
// nearest floats, 14.9 with these, 15.7 with all 24 bits of a float kept.
__device__ __forceinline__ float to_odd_float(double v) {
    const uint64_t u = __double_as_longlong(v);
    const uint32_t hi = static_cast<uint32_t>(u >> 32) | (static_cast<uint32_t>(u) != 0u ? 1u : 0u);
    return static_cast<float>(__longlong_as_double(static_cast<uint64_t>(hi) << 32));
}

}  // namespace nmm
