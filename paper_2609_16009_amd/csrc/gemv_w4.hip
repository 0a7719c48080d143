// Products with 4-bit weights and group scales on the matrix cores (gfx950):
//   y[m, n] = sum_k x[m, k] * s[n, k / G] * c[n, k],   c = u - z (integers) or an e2m1 value
//
// The weight is what has to be read, a quarter of a 16-bit one's bytes, so at few rows of x the work is to
// keep enough of it in flight and to widen it in the shadow of its loads:
//  * A workgroup owns 64 NT rows of the weight, 16 NT a wave, and a slice of K.  x's rows of the slice are staged in
//    LDS once, for all waves, and so are the rows' scales and zero points; then each wave streams its rows through a ring
//    of its own, D slots of 256 k (128 bytes, one cache line, of each row) in flight, with no barrier in the loop.
//    Loads go straight to LDS, 8 rows x 128 bytes each; chunks of 16 bytes are permuted within a row so that
//    fragment reads hit every bank once.
//  * Chunk i of a row is 32 k, one step of v_mfma_f32_16x16x32 and one group at most: lane (g, j) reads dword g
//    of row j, 8 codes, and widens them exactly.  An integer code u is, as the e4m3 byte u, the number
//    u * 2^-9 (subnormals and the first binade of e4m3 are one uniform grid), so v_cvt_scalef32_pk_{bf16,f16}_fp8 with
//    a scale of 2^9 yields u; e2m1 has v_cvt_scalef32_pk_{bf16,f16}_fp4.  No weight is ever rounded: the scale is applied
//    to the group's fp32 sum.
//  * Zero points: sum_k x (u - z) = sum_k x u - z sum_k x, the second sum by one more MFMA with ones per
//    step, shared by the wave's row tiles.
//  * x is the A operand and the weight the B operand, so that a lane's four sums belong to one weight row
//    and share its scale.
//  * K is split over workgroups to fill the chip; the last to finish adds the slices in slice order (handoff.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "handoff.h"
#include "nmm_internal.h"

namespace nmm {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRsrcWord3 = 0x00020000;
constexpr int kLoadNT = 2;
constexpr int kDevice = 16;                 // sc1: device scope (handoff.h)
constexpr uint32_t kOutOfRange = 0x80000000u;
constexpr int kSlotK = 256;                 // k of a slot
constexpr int kSteps = kSlotK / 32;
constexpr int kMaxGroups = 64;              // groups of a K-slice (their scales lie in LDS)
constexpr int kMaxRows = 32;                // rows of x per block
constexpr int kWaves4 = 4;
// Slots of a K-slice at most: what x's rows of it may take of LDS (8 KB a row of x up to 4 rows, 32 KB in all up to 16
// rows, 64 KB for 32).
constexpr int max_slots(int xr) { return xr <= 4 ? 16 : xr == 8 ? 8 : 4; }

struct W4Params {
    const uint16_t* x;
    int64_t ldx;
    const uint8_t* w;
    const uint8_t* scales;
    const uint8_t* zeros;     // or NULL: 8
    int64_t lds, ldz;         // groups per row
    float* y;
    int64_t ldy;
    float* part;              // [tile][slice][rows of x][16 NT]
    unsigned* tickets;
    uint32_t row_bytes, w_extent;
    int M, K, N, groups, lg_group;
    int row_blocks, mblocks, ks, slots_per_slice, slots;
};

template <int DT>
__device__ __forceinline__ f32x4 mfma(i32x4 a, i32x4 b, f32x4 c) {
    if constexpr (DT == NMM_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The values of 8 codes, k ascending.
template <int DT, bool MX>
__device__ __forceinline__ i32x4 widen(uint32_t q) {
    i32x4 r;
    if constexpr (MX) {
        if constexpr (DT == NMM_BF16) {
            r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, 1.0f, 0));
            r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, 1.0f, 1));
            r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, 1.0f, 2));
            r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(q, 1.0f, 3));
        } else {
            r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, 1.0f, 0));
            r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, 1.0f, 1));
            r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, 1.0f, 2));
            r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(q, 1.0f, 3));
        }
    } else {
        const uint32_t even = q & 0x0F0F0F0Fu, odd = (q >> 4) & 0x0F0F0F0Fu;
        const uint32_t lo = __builtin_amdgcn_perm(odd, even, 0x05010400u), hi = __builtin_amdgcn_perm(odd, even, 0x07030602u);
        if constexpr (DT == NMM_BF16) {
            r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
            r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
            r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
            r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
        } else {
            r[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false));
            r[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true));
            r[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false));
            r[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true));
        }
    }
    return r;
}

template <int DT, bool MX>
__device__ __forceinline__ float scale_value(const uint8_t* s) {
    if constexpr (MX) {
        // 2^(b - 127): b = 0 is a subnormal fp32, 255 NaN
        const uint32_t b = *s;
        return b == 255u ? __uint_as_float(0x7FC00000u) : b == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23);
    } else if constexpr (DT == NMM_BF16) {
        return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(s)) << 16);
    } else {
        return float(*reinterpret_cast<const _Float16*>(s));
    }
}

// XR: rows of x staged (1, 2, 4, 8, 16, 32); NT: 16-row tiles of the weight per wave; D: slots in flight (2 to 4); GS:
// steps of a group within a slot (1, 2, 4, or 8 for groups of 256 k and more).
template <int DT, bool MX, int XR, int NT, int D, int GS>
__global__ __launch_bounds__(64 * kWaves4) void w4_kernel(const W4Params p) {
    constexpr int NW = kWaves4;
    constexpr int MT = XR > 16 ? 2 : 1;
    constexpr int kWLoads = 2 * NT, kSlotBytes = kWLoads * 1024;
    static_assert((D - 1) * kWLoads < 64, "vmcnt holds 6 bits");
    constexpr int kScaleSize = MX ? 1 : 2;
    constexpr int kRows = 16 * NT * NW;
    __shared__ __attribute__((aligned(256))) uint8_t xs_buf[XR * max_slots(XR) * kSlotK * 2];
    __shared__ __attribute__((aligned(128))) uint8_t ring0[NW * kSlotBytes];
    __shared__ __attribute__((aligned(128))) uint8_t ring1[NW * kSlotBytes];
    __shared__ __attribute__((aligned(128))) uint8_t ring2[D > 2 ? NW * kSlotBytes : 16];
    __shared__ __attribute__((aligned(128))) uint8_t ring3[D > 3 ? NW * kSlotBytes : 16];
    // a row's scales, padded to an odd number of dwords so that 16 rows of one group lie in 16 banks
    constexpr int kScalePitch = kMaxGroups * kScaleSize + 4, kZeroPitch = MX ? 4 : kMaxGroups + 4;
    __shared__ __attribute__((aligned(16))) uint8_t sc[kRows * kScalePitch];
    __shared__ __attribute__((aligned(16))) uint8_t zp[MX ? 16 : kRows * kZeroPitch];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (NW - 1);
    const int g = lane >> 4, j = lane & 15;

    // the row blocks of x over one block of weight rows sit 8 workgroup ids apart, on one XCD
    const int per_rb = p.mblocks * p.ks;
    const int bid = static_cast<int>(blockIdx.x);
    const int rb = (bid & 7) + 8 * (bid / (8 * per_rb));
    const int rest = (bid >> 3) % per_rb;
    const int slice = rest / p.mblocks, mb = rest - slice * p.mblocks;
    if (rb >= p.row_blocks) return;
    const int n0 = rb * kRows, nw = n0 + wave * 16 * NT, m0 = mb * XR;
    const int mrows = min(XR, p.M - m0);
    const int slot0 = slice * p.slots_per_slice, slot1 = min(p.slots, slot0 + p.slots_per_slice);
    const int n_slots = slot1 - slot0;
    const int k_begin = slot0 * kSlotK;
    const int group0 = k_begin >> p.lg_group;

    const __amdgpu_buffer_rsrc_t wr =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.w), (short)0, (int)p.w_extent, kRsrcWord3);
    const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint16_t*>(p.x + int64_t(m0) * p.ldx), (short)0,
        int(uint32_t((int64_t(mrows - 1) * p.ldx + (p.K + 7) / 8 * 8) * 2)), kRsrcWord3);

    // Weight load q of a slot: rows 8 q + lane / 8, slot lane % 8 of the row holds its chunk (lane % 8) ^ (row / 2 % 8).
    uint32_t woff[kWLoads];
    int wk[2];                                   // the chunk's first k: rows 8 q, q even and odd
#pragma unroll
    for (int q = 0; q < kWLoads; ++q) {
        const int r = 8 * q + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
        if (q < 2) wk[q] = 32 * c;
        woff[q] = nw + r < p.N ? uint32_t(nw + r) * p.row_bytes + 16u * c : kOutOfRange;
    }
    auto load_slot = [&](int slot, uint8_t* ring) {
        uint8_t* const dst = ring + wave * kSlotBytes;
        const int k0 = slot * kSlotK;
        const int left = slot < slot1 ? p.K - k0 : 0;        // a slot past the slice loads nothing
#pragma unroll
        for (int q = 0; q < kWLoads; ++q) {
            const uint32_t o = wk[q & 1] < left ? woff[q] + uint32_t(k0 / 2) : kOutOfRange;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(dst + q * 1024), 16, o, 0, 0, kLoadNT);
        }
    };
    // The slice's scales and zero points (rows past N: the last one's; without zero points all are 8) are loaded first, to
    // registers, then x and the ring's first slots, so that all of it is in flight at once.
    constexpr int kPer = 64 * NW / kRows, kTimes = kMaxGroups / kPer;         // threads per row, groups per thread
    const int n_groups = min(p.groups - group0, ((slot1 * kSlotK - 1) >> p.lg_group) - group0 + 1);
    const int sr = tid / kPer, sg = tid % kPer;
    uint32_t sreg[kTimes], zreg[kTimes];
    {
        const int64_t n = min(n0 + sr, p.N - 1);
        const uint8_t* const s8 = p.scales + (n * p.lds + group0) * kScaleSize;
        const uint8_t* const z8 = MX || !p.zeros ? s8 : p.zeros + n * p.ldz + group0;
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (i * kPer >= n_groups) break;
            const int gr = min(i * kPer + sg, n_groups - 1);
            if constexpr (MX) {
                sreg[i] = s8[gr];
            } else {
                sreg[i] = reinterpret_cast<const uint16_t*>(s8)[gr];
                if (p.zeros) zreg[i] = z8[gr];
            }
        }
    }
    // x: half a row's slot (32 chunks of 8 k) in half a load: unit u is slot u % n_slots of row u / n_slots; slot c of
    // row r holds chunk c ^ (r % 16), so that 16 rows of one chunk lie in 16 columns of LDS.
    const int units = XR * n_slots;
    for (int u0 = 2 * wave; u0 < units; u0 += 2 * NW) {
        const int u = u0 + (lane >> 5);
        const int r = u / n_slots, sl = u - r * n_slots;
        const int k = (slot0 + sl) * kSlotK + 8 * ((lane & 31) ^ (r & 15));
        const uint32_t o = u < units && r < mrows && k < p.K ? uint32_t((int64_t(r) * p.ldx + k) * 2) : kOutOfRange;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)(xs_buf + u0 * 512), 16, o, 0, 0, 0);
    }
    load_slot(slot0, ring0);
    load_slot(slot0 + 1, ring1);
    if constexpr (D > 2) load_slot(slot0 + 2, ring2);
    if constexpr (D > 3) load_slot(slot0 + 3, ring3);
#pragma unroll
    for (int i = 0; i < kTimes; ++i) {
        if (i * kPer >= n_groups) break;
        const int gr = i * kPer + sg;
        if constexpr (MX) {
            sc[sr * kScalePitch + gr] = uint8_t(sreg[i]);
        } else {
            *reinterpret_cast<uint16_t*>(sc + sr * kScalePitch + 2 * gr) = uint16_t(sreg[i]);
            zp[sr * kZeroPitch + gr] = p.zeros ? uint8_t(zreg[i]) : uint8_t(8);
        }
    }
    // (x has landed once at most the weight's loads are outstanding; those stay in flight)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(D * kWLoads) : "memory");
    // what a chunk that K ends in holds past K is cleared
    if (p.K % 8 && p.K > k_begin && p.K <= slot1 * kSlotK) {
        const int c = (p.K - k_begin) / 8;
        for (int i = tid; i < XR * 8; i += 64 * NW) {
            const int r = i / 8, e = i % 8;
            if (e >= p.K % 8)
                *reinterpret_cast<uint16_t*>(xs_buf + (r * n_slots + c / 32) * 512 + (((c % 32) ^ (r & 15)) << 4) + 2 * e) = 0;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");      // (the weight's loads stay in flight)
    }

    f32x4 sum[NT][MT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sum[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int jx = XR < 16 ? (j & (XR - 1)) : j;
    const i32x4 ones = DT == NMM_BF16 ? i32x4{0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80}
                                      : i32x4{0x3C003C00, 0x3C003C00, 0x3C003C00, 0x3C003C00};
    const uint8_t* const sc_row = sc + (wave * 16 * NT + j) * kScalePitch;
    const uint8_t* const zp_row = zp + (MX ? 0 : (wave * 16 * NT + j) * kZeroPitch);

    auto consume = [&](const uint8_t* ring, int sl) {
        // the slot has landed once at most the younger slots' loads are outstanding (loads complete in order)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * kWLoads) : "memory");
        const uint8_t* const src = ring + wave * kSlotBytes;
        const int k0 = (slot0 + sl) * kSlotK;
        const int gr0 = (k0 >> p.lg_group) - group0;
        // all that the slot's steps read, first
        i32x4 xf[kSteps][MT];
        uint32_t q[kSteps][NT];
        float sv[kSteps / GS][NT], zv[kSteps / GS][NT];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
                q[i][t] = *reinterpret_cast<const uint32_t*>(src + (16 * t + j) * 128 + ((i ^ ((j >> 1) & 7)) << 4) + 4 * g);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int r = 16 * mt + jx;
                xf[i][mt] = *reinterpret_cast<const i32x4*>(xs_buf + (r * n_slots + sl) * 512 + (((4 * i + g) ^ (r & 15)) << 4));
            }
            if (i % GS == GS - 1) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const int gr = gr0 + i / GS;
                    sv[i / GS][t] = scale_value<DT, MX>(sc_row + 16 * t * kScalePitch + gr * kScaleSize);
                    if constexpr (!MX) zv[i / GS][t] = float(zp_row[16 * t * kZeroPitch + gr]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        f32x4 acc[NT][MT], xs[MT];
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            if (i % GS == 0) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    xs[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int t = 0; t < NT; ++t) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
            }
            if constexpr (!MX) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) xs[mt] = mfma<DT>(xf[i][mt], ones, xs[mt]);
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const i32x4 wf = widen<DT, MX>(q[i][t]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc[t][mt] = mfma<DT>(xf[i][mt], wf, acc[t][mt]);
            }
            if (i % GS == GS - 1) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    // (a group that starts past K has no scale)
                    const float s = k0 + 32 * (i / GS * GS) < p.K ? sv[i / GS][t] : 0.f;
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float a = MX ? acc[t][mt][e] : __builtin_fmaf(-zv[i / GS][t], xs[mt][e], acc[t][mt][e]);
                            sum[t][mt][e] = __builtin_fmaf(s, a, sum[t][mt][e]);
                        }
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (read before the ring is loaded again)
    };
    for (int sl = 0; sl < n_slots; sl += D) {
        consume(ring0, sl);
        load_slot(slot0 + sl + D, ring0);
        if (sl + 1 < n_slots) consume(ring1, sl + 1);
        load_slot(slot0 + sl + D + 1, ring1);
        if constexpr (D > 2) {
            if (sl + 2 < n_slots) consume(ring2, sl + 2);
            load_slot(slot0 + sl + D + 2, ring2);
        }
        if constexpr (D > 3) {
            if (sl + 3 < n_slots) consume(ring3, sl + 3);
            load_slot(slot0 + sl + D + 3, ring3);
        }
    }
    __builtin_amdgcn_s_waitcnt(0);        // (no load may write LDS after the workgroup has left)

    // lane (g, j) holds m = 4 g + e, n = j of each tile
    const int64_t tile = int64_t(rb) * p.mblocks + mb;
    constexpr int kPart = XR * kRows;
    if (p.ks == 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int m = 16 * mt + 4 * g + e, n = nw + 16 * t + j;
                    if (m < mrows && n < p.N) p.y[int64_t(m0 + m) * p.ldy + n] = sum[t][mt][e];
                }
        return;
    }
    const __amdgpu_buffer_rsrc_t pr = __builtin_amdgcn_make_buffer_rsrc(p.part + tile * p.ks * kPart, (short)0,
                                                                        int(uint32_t(p.ks) * kPart * 4u), kRsrcWord3);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = 16 * mt + 4 * g + e;
                if (m < mrows)
                    __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(sum[t][mt][e]), pr,
                                                          uint32_t(slice * kPart + m * kRows + (wave * NT + t) * 16 + j) * 4u, 0, kDevice);
            }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0) s_last = arrive(p.tickets + tile, unsigned(p.ks));
    __syncthreads();
    if (!s_last) return;
    constexpr int kBatch = 8;
    for (int o = tid; o < kRows * mrows; o += 64 * NW) {
        float v = 0.f;
        for (int q0 = 0; q0 < p.ks; q0 += kBatch) {
            float u[kBatch];
#pragma unroll
            for (int q = 0; q < kBatch; ++q)
                u[q] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                    pr, q0 + q < p.ks ? uint32_t((q0 + q) * kPart + o) * 4u : kOutOfRange, 0, kDevice));
#pragma unroll
            for (int q = 0; q < kBatch; ++q) v += u[q];
        }
        const int m = o / kRows, n = n0 + o - m * kRows;
        if (n < p.N) p.y[int64_t(m0 + m) * p.ldy + n] = v;
    }
}

// ---------------------------------------------------------------------------------------------
// The partition.
// ---------------------------------------------------------------------------------------------
struct W4Plan {
    int xr = 1, nt = 1;
    int row_blocks = 1, mblocks = 1, ks = 1, slots = 1, slots_per_slice = 1;
    int64_t grid = 0;
    size_t ws_bytes = 0;
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kLim = int64_t(1) << 31;
constexpr int kTargetGrid = 512;

nmm_status plan_w4(int64_t M, int64_t K, int64_t N, int64_t group, W4Plan* out) {
    W4Plan q;
    if (M <= 0 || K <= 0 || N <= 0) {
        *out = q;
        return NMM_OK;
    }
    q.xr = M <= 1 ? 1 : M <= 2 ? 2 : M <= 4 ? 4 : M <= 8 ? 8 : M <= 16 ? 16 : 32;
    q.mblocks = static_cast<int>(cdiv(M, q.xr));
    q.nt = 1;
    const int rows = 16 * kWaves4 * q.nt;
    q.row_blocks = static_cast<int>(cdiv(N, rows));
    q.slots = static_cast<int>(cdiv(K, kSlotK));
    // slices: enough workgroups, but at least four slots each, and no more of K than LDS holds x's rows and the scales of
    const int64_t tiles = int64_t(q.row_blocks) * q.mblocks;
    const int64_t most = std::min<int64_t>(max_slots(q.xr), std::max<int64_t>(1, kMaxGroups * group / kSlotK));
    int64_t ks = std::max<int64_t>(1, std::min<int64_t>(kTargetGrid / std::max<int64_t>(1, tiles), q.slots / 4));
    ks = std::max(ks, cdiv(q.slots, most));
    const int64_t per = cdiv(q.slots, ks);
    q.slots_per_slice = static_cast<int>(per);
    q.ks = static_cast<int>(cdiv(q.slots, per));
    q.grid = cdiv(q.row_blocks, 8) * 8 * q.mblocks * q.ks;
    if (q.grid >= (int64_t(1) << 32) / (64 * kWaves4)) return NMM_ERR_SHAPE;
    if (q.ks > 1) {
        if (tiles > kMaxTickets) return NMM_ERR_SHAPE;
        q.ws_bytes = size_t(kTicketBytes) + size_t(tiles) * q.ks * q.xr * rows * 4;
    }
    *out = q;
    return NMM_OK;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int DT, bool MX, int XR, int NT, int D>
void launch_gs(const W4Params& p, const W4Plan& q, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(q.grid)), block(64 * kWaves4);
    if constexpr (MX) {
        hipLaunchKernelGGL((w4_kernel<DT, true, XR, NT, D, 1>), grid, block, 0, s, p);
    } else {
        switch (p.lg_group) {
            case 5: hipLaunchKernelGGL((w4_kernel<DT, false, XR, NT, D, 1>), grid, block, 0, s, p); break;
            case 6: hipLaunchKernelGGL((w4_kernel<DT, false, XR, NT, D, 2>), grid, block, 0, s, p); break;
            case 7: hipLaunchKernelGGL((w4_kernel<DT, false, XR, NT, D, 4>), grid, block, 0, s, p); break;
            default: hipLaunchKernelGGL((w4_kernel<DT, false, XR, NT, D, 8>), grid, block, 0, s, p); break;
        }
    }
}

template <int DT, bool MX>
void launch_xr(const W4Params& p, const W4Plan& q, hipStream_t s) {
    switch (q.xr) {
        case 1: launch_gs<DT, MX, 1, 1, 4>(p, q, s); break;
        case 2: launch_gs<DT, MX, 2, 1, 4>(p, q, s); break;
        case 4: launch_gs<DT, MX, 4, 1, 4>(p, q, s); break;
        case 8: launch_gs<DT, MX, 8, 1, 3>(p, q, s); break;
        case 16: launch_gs<DT, MX, 16, 1, 3>(p, q, s); break;
        default: launch_gs<DT, MX, 32, 1, 3>(p, q, s); break;
    }
}

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_gemv_w4_workspace_size(int64_t M, int64_t K, int64_t N, int64_t group) {
    if (M < 0 || K < 0 || N < 0 || M >= kLim || K >= kLim || N >= kLim || group < 32 || (group & (group - 1))) return 0;
    W4Plan q;
    return plan_w4(M, K, N, group, &q) == NMM_OK ? q.ws_bytes : 0;
}

nmm_status nmm_gemv_w4(int64_t M, int64_t K, int64_t N, nmm_dtype dt, nmm_w4_format format, int64_t group, const void* x,
                       int64_t ldx, const void* Wq, int64_t ldwq, const void* scales, int64_t lds, const uint8_t* zeros,
                       int64_t ldz, float* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
    if (dt != NMM_F16 && dt != NMM_BF16) return NMM_ERR_DTYPE;
    if (format != NMM_W4_INT && format != NMM_W4_MX) return NMM_ERR_DTYPE;
    if (M < 0 || K < 0 || N < 0 || M >= kLim || K >= kLim || N >= kLim) return NMM_ERR_SHAPE;
    if (group < 32 || group >= kLim || (group & (group - 1)) || (format == NMM_W4_MX && group != 32)) return NMM_ERR_SHAPE;
    if (format == NMM_W4_MX && zeros) return NMM_ERR_ARG;
    if (M == 0 || N == 0) return NMM_OK;
    if (!y) return NMM_ERR_NULL;
    if (ldy < N || ldy >= kLim) return NMM_ERR_SHAPE;
    if (!aligned(y, 4)) return NMM_ERR_ALIGN;
    GemvArgs a;
    a.M = M; a.K = K; a.N = N; a.dt = dt; a.y = y; a.ldy = ldy;
    if (K == 0) return launch_gemv(a, GemvPlan{}, nullptr, nullptr, stream);
    if (!x || !Wq || !scales) return NMM_ERR_NULL;
    const int64_t groups = cdiv(K, group);
    if (ldx < K || ldx >= kLim || ldwq < cdiv(K, 2) || ldwq >= kLim || lds < groups || lds >= kLim ||
        (zeros && (ldz < groups || ldz >= kLim)))
        return NMM_ERR_SHAPE;
    if (!aligned(x, 16) || !aligned(Wq, 16) || ldx % 8 || ldwq % 16 || !aligned(scales, format == NMM_W4_MX ? 1 : 2))
        return NMM_ERR_ALIGN;
    // buffer offsets are 32-bit: the weight, and the x rows of a block
    const int64_t w_extent = (N - 1) * ldwq + cdiv(K, 32) * 16;
    if (w_extent >= kLim) return NMM_ERR_SHAPE;
    if (((std::min<int64_t>(M, kMaxRows) - 1) * ldx + cdiv(K, 8) * 8) * 2 >= kLim) return NMM_ERR_SHAPE;
    W4Plan q;
    nmm_status st = plan_w4(M, K, N, group, &q);
    if (st != NMM_OK) return st;
    st = validate_workspace(workspace, workspace_bytes, q.ws_bytes);
    if (st != NMM_OK) return st;
    W4Params p{};
    p.x = static_cast<const uint16_t*>(x);
    p.ldx = ldx;
    p.w = static_cast<const uint8_t*>(Wq);
    p.scales = static_cast<const uint8_t*>(scales);
    p.zeros = zeros;
    p.lds = lds;
    p.ldz = ldz;
    p.y = y;
    p.ldy = ldy;
    if (q.ks > 1) {
        p.tickets = static_cast<unsigned*>(workspace);
        p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
    }
    p.row_bytes = static_cast<uint32_t>(ldwq);
    p.w_extent = static_cast<uint32_t>(w_extent);
    p.M = static_cast<int>(M);
    p.K = static_cast<int>(K);
    p.N = static_cast<int>(N);
    p.groups = static_cast<int>(groups);
    while ((int64_t(1) << p.lg_group) < group) ++p.lg_group;
    p.row_blocks = q.row_blocks;
    p.mblocks = q.mblocks;
    p.ks = q.ks;
    p.slots_per_slice = q.slots_per_slice;
    p.slots = q.slots;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool mx = format == NMM_W4_MX;
    if (dt == NMM_BF16) mx ? launch_xr<NMM_BF16, true>(p, q, s) : launch_xr<NMM_BF16, false>(p, q, s);
    else mx ? launch_xr<NMM_F16, true>(p, q, s) : launch_xr<NMM_F16, false>(p, q, s);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
