// Rows of the latent cache written and read for many tokens at once.
//
//   entry[t] = bf16([RMSNorm(c) * gamma | RoPE(k, positions[t])])        src[t] = [c | k]
//   8 bits:   per block of 32 latents the least e >= -117 with max |v| <= 448 * 2^e; code = e4m3(v * 2^-e)
//
// The entry is rounded to bf16 first, so an 8-bit row holds the codes of the bf16 row that this call would have written
// for the same token.  v * 2^-e is exact, so a code has one rounding.  bf16() is the nearest float of the 64-bit value and
// of that the nearest bf16 number, as casts of a double to bf16 commonly are: 9 of 10^6 of RMSNorm's and RoPE's values lie so near to
// a tie that the float is the tie and goes to even (the float rounded to odd instead, which rounds once: 14.9 us for 14.5).
// fp32 arithmetic (nmm_mla_kv_update) moves about as many entries, others, and where one moves so may its 8-bit code, a whole step.
//
//  * Writing: a wave owns a token, a lane eight latents, four lanes a scale block, whose maximum meets by
//    two DPP exchanges; the sum of squares is a butterfly over the wave, and RMSNorm and RoPE are in fp64 up to
//    the float that the entry is rounded from.  Lanes below rope / 2 take a RoPE
//    pair each.  Nothing leaves the wave, so tokens need no barrier and any number of them fills the chip.
//  * Reading: a thread owns 16 bytes of an output row, so stores are whole lines and the loads of a row
//    are contiguous too.
// Bound by bytes for many rows and by one chain of round trips for few: 40001 8-bit rows of 656 bytes read into bf16
// ones in 16.4 us (72 MB, 4.4 TB/s, against 5.1 of a large copy) with 216 MB in turn, which the last-level cache holds, and 23.4 with
// 1 GiB; 8192 rows written from fp32 and read back 14.6 us (two launches, 39 MB; 17.6 with 1 GiB in turn), of which RMSNorm
// and RoPE in fp64 are 0.9; 64 rows 5.4 us for both launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "bf16_cast.h"
#include "latent_row.h"
#include "nmm_internal.h"
#include "rope.h"

namespace nmm {
namespace {

constexpr int kCacheThreads = 256;
constexpr int kTokensPerGroup = kCacheThreads / 64;

struct WriteParams {
    const void* src;
    int64_t ld_src;            // elements
    const int64_t* slots;
    const uint16_t* gamma;     // or NULL: no RMSNorm
    const int64_t* positions;  // or NULL: no RoPE
    uint8_t* data;
    int64_t rows, ld;
    double freq_step;
    float eps;
    int tokens, kv, rope;
};

template <int CTRL>
__device__ __forceinline__ float dpp_move(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, false));
}
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

template <int CTRL>
__device__ __forceinline__ double dpp_move(double x) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_mov_dpp(int(uint32_t(u)), CTRL, 0xF, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_mov_dpp(int(uint32_t(u >> 32)), CTRL, 0xF, 0xF, false);
    return __longlong_as_double((uint64_t(hi) << 32) | lo);
}

// The sum over the wave in every lane, in a fixed order: quads, half rows, rows, then across rows.
__device__ __forceinline__ double sum64(double x) {
    x += dpp_move<0xB1>(x);
    x += dpp_move<0x4E>(x);
    x += dpp_move<0x141>(x);
    x += dpp_move<0x140>(x);
    uint64_t u = __double_as_longlong(x);
    u32x2 lo = __builtin_amdgcn_permlane16_swap(uint32_t(u), uint32_t(u), false, false);
    u32x2 hi = __builtin_amdgcn_permlane16_swap(uint32_t(u >> 32), uint32_t(u >> 32), false, false);
    x = __longlong_as_double((uint64_t(hi[0]) << 32) | lo[0]) + __longlong_as_double((uint64_t(hi[1]) << 32) | lo[1]);
    u = __double_as_longlong(x);
    lo = __builtin_amdgcn_permlane32_swap(uint32_t(u), uint32_t(u), false, false);
    hi = __builtin_amdgcn_permlane32_swap(uint32_t(u >> 32), uint32_t(u >> 32), false, false);
    return __longlong_as_double((uint64_t(hi[0]) << 32) | lo[0]) + __longlong_as_double((uint64_t(hi[1]) << 32) | lo[1]);
}

// x^(-1/2): the fp32 instruction and one Newton step in fp64 (1e-14), or in fp64 altogether outside fp32's range.
__device__ __forceinline__ double inverse_root(double x) {
    if (!(x > 1e-30 && x < 1e30)) return 1.0 / __builtin_sqrt(x);
    const double y = double(__builtin_amdgcn_rsqf(float(x)));
    return y * (1.5 - 0.5 * x * y * y);
}

__device__ __forceinline__ float bf16_up(uint32_t bits) { return __uint_as_float(bits << 16); }

template <bool SRC_BF16, bool E4M3>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(const WriteParams p) {
    const int lane = threadIdx.x & 63;
    const int t = static_cast<int>(blockIdx.x) * kTokensPerGroup + (threadIdx.x >> 6);
    if (t >= p.tokens) return;
    const int64_t slot = p.slots[t];
    const int64_t pos = p.positions ? p.positions[t] : 0;
    const int c = 8 * lane;
    const bool has = c < p.kv;
    const bool pair = lane < p.rope / 2;
    float v[8], k0 = 0.f, k1 = 0.f;
    if constexpr (SRC_BF16) {
        const uint16_t* s = static_cast<const uint16_t*>(p.src) + int64_t(t) * p.ld_src;
        uint4 u{0, 0, 0, 0};
        if (has) u = *reinterpret_cast<const uint4*>(s + c);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = bf16_up(w[i] & 0xFFFFu);
            v[2 * i + 1] = bf16_up(w[i] >> 16);
        }
        if (pair) {
            const uint32_t w2 = *reinterpret_cast<const uint32_t*>(s + p.kv + 2 * lane);
            k0 = bf16_up(w2 & 0xFFFFu);
            k1 = bf16_up(w2 >> 16);
        }
    } else {
        const float* s = static_cast<const float*>(p.src) + int64_t(t) * p.ld_src;
        float4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
        if (has) {
            a = *reinterpret_cast<const float4*>(s + c);
            b = *reinterpret_cast<const float4*>(s + c + 4);
        }
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        if (pair) {
            const float2 w = *reinterpret_cast<const float2*>(s + p.kv + 2 * lane);
            k0 = w.x;
            k1 = w.y;
        }
    }
    if (p.gamma) {
        uint4 g{0, 0, 0, 0};
        if (has) g = *reinterpret_cast<const uint4*>(p.gamma + c);
        // in fp64: an entry that fp32 moves over a boundary between two bf16 numbers may move a whole step of its 8-bit code
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += double(v[i]) * double(v[i]);
        const double inv = inverse_root(sum64(ss) / double(p.kv) + double(p.eps));
        const uint32_t w[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = float(double(v[2 * i]) * inv * double(bf16_up(w[i] & 0xFFFFu)));
            v[2 * i + 1] = float(double(v[2 * i + 1]) * inv * double(bf16_up(w[i] >> 16)));
        }
    }
    if (slot < 0 || slot >= p.rows) return;        // (checked here, so that the row is loaded beside its slot)
    uint8_t* const row = p.data + slot * p.ld;
    const int64_t rope_at = E4M3 ? p.kv + kScaleBytes : 2 * p.kv;
    if (pair) {
        float r0 = k0, r1 = k1;
        if (p.positions) {
            double sn, cs;
            rope_sincos64(p.freq_step, pos, lane, &sn, &cs);
            r0 = float(double(k0) * cs - double(k1) * sn);
            r1 = float(double(k0) * sn + double(k1) * cs);
        }
        *reinterpret_cast<uint32_t*>(row + rope_at + 4 * lane) = uint32_t(to_bf16_bits(r0)) | (uint32_t(to_bf16_bits(r1)) << 16);
    }
    uint32_t h[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = to_bf16_bits(v[i]);
    if constexpr (!E4M3) {
        if (has)
            *reinterpret_cast<uint4*>(row + 2 * c) =
                uint4{h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16)};
    } else {
        // the block's largest finite magnitude, over the quad's 32 values (a whole quad has values or none)
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = bf16_up(h[i]);
            const bool finite = (h[i] & 0x7F80u) != 0x7F80u;
            top = finite ? fmaxf(top, fabsf(v[i])) : top;
            // e4m3 has no infinity: what is not finite is kept as NaN
            if (!finite) v[i] = __uint_as_float(0x7FC00000u);
        }
        top = fmaxf(top, dpp_move<0xB1>(top));
        top = fmaxf(top, dpp_move<0x4E>(top));
        // top = 1.m * 2^x against 448 = 1.75 * 2^8
        const uint32_t bits = __float_as_uint(top);
        const int e = max(int(bits >> 23) - 127 - 8 + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0), kMinScaleExp);
        const float inv = __uint_as_float(uint32_t(127 - e) << 23);
        if (has) {
            int lo = 0, hi = 0;
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0] * inv, v[1] * inv, lo, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2] * inv, v[3] * inv, lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4] * inv, v[5] * inv, hi, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6] * inv, v[7] * inv, hi, true);
            *reinterpret_cast<uint2*>(row + c) = uint2{uint32_t(lo), uint32_t(hi)};
        }
        // the scale bytes, those past kv_lora / 32 as 127 (a scale of one): lane 4 b holds block b's
        if ((lane & 3) == 0) row[p.kv + (lane >> 2)] = static_cast<uint8_t>(has ? e + 127 : 127);
    }
}

struct ReadParams {
    const uint8_t* data;
    int64_t rows, ld;
    const int64_t* slots;
    uint16_t* out;
    int64_t ldo;               // elements
    int64_t pieces;            // tokens * per_row
    int kv, per_row;           // 16-byte pieces of an output row
};

template <bool E4M3>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(const ReadParams p) {
    const int64_t i = int64_t(blockIdx.x) * kCacheThreads + threadIdx.x;
    if (i >= p.pieces) return;
    const int64_t t = i / p.per_row;
    const int c = 8 * static_cast<int>(i - t * p.per_row);
    const int64_t slot = p.slots[t];
    if (slot < 0 || slot >= p.rows) return;
    const uint8_t* row = p.data + slot * p.ld;
    uint4 v;
    if (E4M3 && c < p.kv) {
        const uint2 q = *reinterpret_cast<const uint2*>(row + c);
        const float s = scale_of(row[p.kv + c / kScaleBlock]);
        const uint2 a = dequant4(q.x, s), b = dequant4(q.y, s);
        v = uint4{a.x, a.y, b.x, b.y};
    } else {
        v = *reinterpret_cast<const uint4*>(row + (E4M3 ? p.kv + kScaleBytes + 2 * (c - p.kv) : 2 * c));
    }
    *reinterpret_cast<uint4*>(p.out + t * p.ldo + c) = v;
}

constexpr int64_t kLim = int64_t(1) << 31;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_latent_cache_row_bytes(nmm_cache_format format, int64_t kv_lora, int64_t rope) {
    if (format != NMM_CACHE_BF16 && format != NMM_CACHE_E4M3) return 0;
    if (kv_lora < kScaleBlock || kv_lora > kLatentMax || kv_lora % kScaleBlock) return 0;
    if (rope < 0 || rope > kLatentRopeMax || rope % 8) return 0;
    return static_cast<size_t>(latent_row_bytes(format, kv_lora, rope));
}

nmm_status nmm_latent_cache_write(const nmm_latent_cache* cache, const nmm_cache_entries* entries, void* stream) {
    if (!cache || !entries) return NMM_ERR_NULL;
    const nmm_latent_cache& c = *cache;
    const nmm_cache_entries& e = *entries;
    const nmm_status st = validate_latent_cache(c);
    if (st != NMM_OK) return st;
    if (e.src_type != NMM_SRC_F32 && e.src_type != NMM_SRC_BF16) return NMM_ERR_DTYPE;
    if (e.tokens < 0 || e.tokens >= kLim) return NMM_ERR_SHAPE;
    const int64_t piece = e.src_type == NMM_SRC_F32 ? 4 : 8;   // elements of 16 bytes
    if (e.ld_src < c.kv_lora + c.rope || e.ld_src >= kLim) return NMM_ERR_SHAPE;
    if (e.gamma && (!std::isfinite(e.eps) || e.eps < 0.f)) return NMM_ERR_ARG;
    if (e.positions && (!std::isfinite(e.rope_theta) || e.rope_theta <= 0.f)) return NMM_ERR_ARG;
    if (e.tokens == 0) return NMM_OK;
    if (!e.src || !e.slots || (!c.data && c.rows > 0)) return NMM_ERR_NULL;
    if (e.ld_src % piece || !aligned(e.src, 16) || !aligned(e.gamma, 16) || !aligned(e.slots, 8) || !aligned(e.positions, 8))
        return NMM_ERR_ALIGN;
    if (c.rows == 0) return NMM_OK;
    WriteParams p{};
    p.src = e.src;
    p.ld_src = e.ld_src;
    p.slots = e.slots;
    p.gamma = static_cast<const uint16_t*>(e.gamma);
    p.positions = e.positions;
    p.data = static_cast<uint8_t*>(c.data);
    p.rows = c.rows;
    p.ld = c.ld;
    p.freq_step = c.rope > 0 && e.positions ? std::pow(double(e.rope_theta), -2.0 / double(c.rope)) : 1.0;
    p.eps = e.eps;
    p.tokens = static_cast<int>(e.tokens);
    p.kv = static_cast<int>(c.kv_lora);
    p.rope = static_cast<int>(c.rope);
    const dim3 grid(static_cast<uint32_t>((e.tokens + kTokensPerGroup - 1) / kTokensPerGroup)), block(kCacheThreads);
    // a launch has fewer than 2^32 threads
    if (int64_t(grid.x) * kCacheThreads >= (int64_t(1) << 32)) return NMM_ERR_SHAPE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf = e.src_type == NMM_SRC_BF16, q8 = c.format == NMM_CACHE_E4M3;
    if (bf && q8) hipLaunchKernelGGL((cache_write_kernel<true, true>), grid, block, 0, s, p);
    else if (bf) hipLaunchKernelGGL((cache_write_kernel<true, false>), grid, block, 0, s, p);
    else if (q8) hipLaunchKernelGGL((cache_write_kernel<false, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((cache_write_kernel<false, false>), grid, block, 0, s, p);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

nmm_status nmm_latent_cache_read(const nmm_latent_cache* cache, int64_t tokens, const int64_t* slots, void* out,
                                 int64_t ldo, void* stream) {
    if (!cache) return NMM_ERR_NULL;
    const nmm_latent_cache& c = *cache;
    const nmm_status st = validate_latent_cache(c);
    if (st != NMM_OK) return st;
    if (tokens < 0 || tokens >= kLim) return NMM_ERR_SHAPE;
    if (ldo < c.kv_lora + c.rope || ldo >= kLim) return NMM_ERR_SHAPE;
    if (tokens == 0) return NMM_OK;
    if (!slots || !out || (!c.data && c.rows > 0)) return NMM_ERR_NULL;
    if (!aligned(out, 16) || ldo % 8 || !aligned(slots, 8)) return NMM_ERR_ALIGN;
    if (c.rows == 0) return NMM_OK;
    ReadParams p{};
    p.data = static_cast<const uint8_t*>(c.data);
    p.rows = c.rows;
    p.ld = c.ld;
    p.slots = slots;
    p.out = static_cast<uint16_t*>(out);
    p.ldo = ldo;
    p.kv = static_cast<int>(c.kv_lora);
    p.per_row = static_cast<int>((c.kv_lora + c.rope) / 8);
    p.pieces = tokens * p.per_row;
    // a launch has fewer than 2^32 threads
    if (p.pieces + kCacheThreads >= (int64_t(1) << 32)) return NMM_ERR_SHAPE;
    const dim3 grid(static_cast<uint32_t>((p.pieces + kCacheThreads - 1) / kCacheThreads)), block(kCacheThreads);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (c.format == NMM_CACHE_E4M3) hipLaunchKernelGGL((cache_read_kernel<true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((cache_read_kernel<false>), grid, block, 0, s, p);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
