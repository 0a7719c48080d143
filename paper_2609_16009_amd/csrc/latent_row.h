// Rows of the latent cache in their two formats, shared by the kernels that write and read them.
//
//   NMM_CACHE_BF16   kv_lora latents, then rope values, bf16
//   NMM_CACHE_E4M3   kv_lora e4m3 codes, kScaleBytes of scale bytes (one per kScaleBlock latents), then
//                    rope values in bf16 (the keys' positions, which 8 bits would blur)
//
// A scale byte b stands for 2^(b - 127).  A power of two costs e4m3 nothing (its precision is relative)
// and makes both directions exact but for the one rounding to e4m3: what a code stands for, 4 significant
// bits times 2^e, is a bf16 value, so attention over 8-bit rows is attention over the bf16 rows that they
// stand for, with no rounding of its own.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nmm.h"

namespace nmm {

constexpr int kLatentMax = 512;      // kv_lora: a multiple of kScaleBlock up to this
constexpr int kLatentRopeMax = 64;   // rope: a multiple of 8 up to this
constexpr int kScaleBlock = 32;
constexpr int kScaleBytes = 16;
constexpr int kMinScaleExp = -117;   // the least code, 2^-9, then stands for 2^-126, the least normal bf16

constexpr int64_t latent_row_bytes(int format, int64_t kv_lora, int64_t rope) {
    return format == NMM_CACHE_E4M3 ? kv_lora + kScaleBytes + 2 * rope : 2 * (kv_lora + rope);
}

// The checks that every call on a latent cache makes.
inline nmm_status validate_latent_cache(const nmm_latent_cache& c) {
    if (c.format != NMM_CACHE_BF16 && c.format != NMM_CACHE_E4M3) return NMM_ERR_DTYPE;
    if (c.kv_lora < kScaleBlock || c.kv_lora > kLatentMax || c.kv_lora % kScaleBlock) return NMM_ERR_SHAPE;
    if (c.rope < 0 || c.rope > kLatentRopeMax || c.rope % 8) return NMM_ERR_SHAPE;
    if (c.rows < 0 || c.rows >= (int64_t(1) << 31)) return NMM_ERR_SHAPE;
    if (c.ld < latent_row_bytes(c.format, c.kv_lora, c.rope) || c.ld >= (int64_t(1) << 31)) return NMM_ERR_SHAPE;
    if (c.ld % 16 || (reinterpret_cast<uintptr_t>(c.data) & 15u)) return NMM_ERR_ALIGN;
    return NMM_OK;
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// 2^(b - 127) of a scale byte.
__device__ __forceinline__ float scale_of(uint32_t b) { return __uint_as_float((b & 255u) << 23); }

// The bf16 values of four e4m3 codes times a power of two (exact).
__device__ __forceinline__ uint2 dequant4(uint32_t codes, float scale) {
    return uint2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}

}  // namespace nmm
