// Products with 4-bit weights and group scales on the matrix cores (gfx950):
//   y[m, n] = sum_k x[m, k] * s[n, k / G] * c[n, k],   c = u - z (integers) or an e2m1 value
//
// The weight is what has to be read, a quarter of a 16-bit one's bytes, so at few rows of x the work is to
// keep enough of it in flight and to widen it in the shadow of its loads:
//  * A workgroup owns 16 rows of the weight per wave (4 to 8 waves) and a slice of K, which its waves stream through a ring
//    in LDS, four slots of 256 k (128 bytes, one cache line, of each row).
//    Loads go straight to LDS, 8 rows x 128 bytes each; chunks of 16 bytes are permuted within a row so that
//    a read of the weight's fragments hits every bank once, and one of 16 rows of x too (8 rows of x lie on half of the banks).  The slice's scales and zero points are staged once, beside the first slots.
//  * Up to 8 rows of x (w4_few_kernel) x's part of the slice is staged once too and each wave goes through its rows on its own,
//    with no barrier in the loop.  More rows (w4_rows_kernel, 16 or 32 at a time) lie in the ring beside the weight, a barrier a
//    slot; a wave there multiplies 32 rows of the weight and half of a slot.
//  * Chunk i of a row is 32 k, one step of v_mfma_f32_16x16x32 and one group at most: lane (g, j) reads dword g
//    of row j, 8 codes, and widens them exactly.  An integer code u is, as the e4m3 byte u, the number
//    u * 2^-9 (subnormals and the first binade of e4m3 are one uniform grid), so v_cvt_scalef32_pk_{bf16,f16}_fp8 with
//    a scale of 2^9 yields u; e2m1 has v_cvt_scalef32_pk_{bf16,f16}_fp4.  No weight is ever rounded: the scale is applied
//    to the group's fp32 sum.
//  * Zero points: sum_k x (u - z) = sum_k x u - z sum_k x.  The second sum is taken once per workgroup while the first slots
//    are on their way (up to 8 rows of x), or by one more MFMA with ones a step.
//  * x is the A operand and the weight the B operand, so that a lane's four sums belong to one weight row
//    and share its scale.
//  * K is split over workgroups to fill the chip; the last to finish adds the slices in slice order (handoff.h).
//
// What bounds it (in a replayed graph; with weights that rotate over 1 GiB, so that none is left in a cache, each within 0.6 us of
// that).  One row of x, K 16384, N 7168, groups of 128: 16.0 us for 60.6 MB, 3.8 TB/s; the same launch without its products 13.9 us,
// without scales and hand-over either 11.7 (5.2 TB/s): half of what is above the loads is widening the codes (7 instructions for
// 512 codes, and a SIMD holds two waves) with their products, half scales and hand-over.  8 rows, K 1536, N 24576, a power of
// two per 32: 9.2 us for 20.9 MB (9.0 without products), six slots a workgroup and so mostly the start.  32 rows of K 16384,
// N 7168: 26 us, 288 TFLOP/s (18.2 without products and hand-over, 14.6 without x's loads either); the MFMAs of x's sums are
// 2.5 us of it.  Of the cycles that LDS is busy 22, 46 and 22 % are bank conflicts by the counters: x's 8 rows account for some
// of the 46, the others have not been traced to their accesses.
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
// Groups of a K-slice at most: their scales lie in LDS, a byte or three each, beside the x rows.
constexpr int max_groups(bool mx, int xr) { return mx || xr <= 4 ? 128 : 64; }
constexpr int kMaxRows = 32;                // rows of x per block
constexpr int kFewRows = 8;                 // up to so many: w4_few_kernel
constexpr int kFewSlots = 16;               // its slots of a K-slice at most (x's rows of them lie in LDS, 8 KB a row)
constexpr int kFewDepth = 4, kRowsDepth = 4;
constexpr int kMaxWaves = 8;
// 16 rows of the weight, a slot of them, in w4_rows_kernel's ring.  (Not 2048 apart: the compiler then reads two tiles by one
// instruction, loses track of which loads that has to wait for and waits for all, 35.3 instead of 28.3 us at
// 32 x 16384 x 7168; the order of the reads is fixed for the same reason.)
constexpr int kTileBytes = 2048 + 16;

struct W4Params {
    const uint16_t* x;
    int64_t ldx;
    const uint8_t* w;
    const uint8_t* scales;
    const uint8_t* zeros;     // or NULL: 8
    int64_t lds, ldz;         // groups per row
    float* y;
    int64_t ldy;
    float* part;              // [tile][slice][rows of x][rows of the weight]
    unsigned* tickets;
    uint32_t row_bytes, w_extent;
    int M, K, N, groups, lg_group;
    int row_blocks, mblocks, ks, slots_per_slice, slots;
    int waves;
};

template <int DT>
__device__ __forceinline__ f32x4 mfma(i32x4 a, i32x4 b, f32x4 c) {
    if constexpr (DT == NMM_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The values of 8 codes, k ascending, or (EVEN_ODD, two instructions fewer) k = 0, 2, 4, 6, 1, 3, 5, 7.
template <int DT, bool MX, bool EVEN_ODD>
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
        const uint32_t lo = EVEN_ODD ? even : __builtin_amdgcn_perm(odd, even, 0x05010400u);
        const uint32_t hi = EVEN_ODD ? odd : __builtin_amdgcn_perm(odd, even, 0x07030602u);
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

template <int DT>
__device__ __forceinline__ float value(uint32_t bits) {
    if constexpr (DT == NMM_BF16) return __uint_as_float(bits << 16);
    else return float(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}

template <int DT, bool MX>
__device__ __forceinline__ float scale_value(uint32_t bits) {
    if constexpr (MX) return bits == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(0x1p-127f, int(bits));      // 2^(b - 127)
    else return value<DT>(bits);
}

// COUNT values of BYTES bytes each, in words where they fill some (the caller's address is a multiple of COUNT * BYTES, or of 4
// where that is more).
template <int COUNT, int BYTES>
__device__ __forceinline__ void read_small(const uint8_t* at, uint32_t (&v)[COUNT]) {
    static_assert(BYTES == 1 || BYTES == 2, "scales and zero points");
    if constexpr (COUNT * BYTES >= 4) {
        constexpr int kPer = 4 / BYTES;
#pragma unroll
        for (int w = 0; w < COUNT / kPer; ++w) {
            const uint32_t u = *reinterpret_cast<const uint32_t*>(at + 4 * w);
#pragma unroll
            for (int i = 0; i < kPer; ++i) v[w * kPer + i] = (u >> (8 * BYTES * i)) & (BYTES == 1 ? 0xFFu : 0xFFFFu);
        }
    } else {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) v[i] = BYTES == 1 ? *(at + i) : *reinterpret_cast<const uint16_t*>(at + 2 * i);
    }
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}

// What a workgroup works on.
struct W4Tile {
    int rows, n0, m0, mrows, rb, mb, slice, slot0, slot1, group0, n_groups;
};

__device__ __forceinline__ bool tile_of(const W4Params& p, int xr, int waves, W4Tile* t) {
    // the row blocks of x over one block of weight rows sit 8 workgroup ids apart, on one XCD
    const int per_rb = p.mblocks * p.ks;
    const int bid = static_cast<int>(blockIdx.x);
    t->rb = (bid & 7) + 8 * (bid / (8 * per_rb));
    const int rest = (bid >> 3) % per_rb;
    t->slice = rest / p.mblocks;
    t->mb = rest - t->slice * p.mblocks;
    t->rows = 16 * waves;
    t->n0 = t->rb * t->rows;
    t->m0 = t->mb * xr;
    t->mrows = min(xr, p.M - t->m0);
    t->slot0 = t->slice * p.slots_per_slice;
    t->slot1 = min(p.slots, t->slot0 + p.slots_per_slice);
    t->group0 = (t->slot0 * kSlotK) >> p.lg_group;
    t->n_groups = min(p.groups - t->group0, ((t->slot1 * kSlotK - 1) >> p.lg_group) - t->group0 + 1);
    return t->rb < p.row_blocks;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t weight_resource(const W4Params& p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(p.w), (short)0, (int)p.w_extent, kRsrcWord3);
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t x_resource(const W4Params& p, const W4Tile& w) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(p.x + int64_t(w.m0) * p.ldx), (short)0,
                                             int(uint32_t((int64_t(w.mrows - 1) * p.ldx + (p.K + 7) / 8 * 8) * 2)), kRsrcWord3);
}

__device__ __forceinline__ void load_x(const __amdgpu_buffer_rsrc_t xr, uint32_t off, uint8_t* dst) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)dst, 16, off, 0, 0, 0);
}

// A wave's 16 rows of the weight, two loads a slot: load q takes rows 8 q + lane / 8, slot lane % 8 of a row holds its
// chunk (lane % 8) ^ (row / 2 % 8).
struct WaveRows {
    uint32_t off[2];
    int k[2];                                    // the chunk's first k
    __device__ __forceinline__ void init(const W4Params& p, int nw, int lane) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int r = 8 * q + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
            k[q] = 32 * c;
            off[q] = nw + r < p.N ? uint32_t(nw + r) * p.row_bytes + 16u * c : kOutOfRange;
        }
    }
    // (left: what of K there is from k0 on; none for a slot past the slice)
    __device__ __forceinline__ void load(const __amdgpu_buffer_rsrc_t wr, int k0, int left, uint8_t* dst) const {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const uint32_t o = k[q] < left ? off[q] + uint32_t(k0 / 2) : kOutOfRange;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(dst + q * 1024), 16, o, 0, 0, kLoadNT);
        }
    }
};

// The slice's scales and zero points, four threads a row (rows past N: the last one's; without zero points all are 8).
template <bool MX, int XR>
struct Scales {
    static constexpr int kMaxGroups = max_groups(MX, XR), kTimes = kMaxGroups / 4;
    static constexpr int kSize = MX ? 1 : 2;
    // a row's scales, padded to an odd number of dwords so that 16 rows of one group lie in 16 banks
    static constexpr int kPitch = kMaxGroups * kSize + 4, kZeroPitch = MX ? 0 : kMaxGroups + 4;
    uint32_t s[kTimes], z[kTimes];
    __device__ __forceinline__ void load(const W4Params& p, const W4Tile& w, int tid) {
        const int64_t n = min(w.n0 + (tid >> 2), p.N - 1);
        const uint8_t* const s8 = p.scales + (n * p.lds + w.group0) * kSize;
        const uint8_t* const z8 = MX || !p.zeros ? s8 : p.zeros + n * p.ldz + w.group0;
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (i * 4 >= w.n_groups) break;
            const int gr = min(i * 4 + (tid & 3), w.n_groups - 1);
            if constexpr (MX) {
                s[i] = s8[gr];
            } else {
                s[i] = reinterpret_cast<const uint16_t*>(s8)[gr];
                if (p.zeros) z[i] = z8[gr];
            }
        }
    }
    __device__ __forceinline__ void store(const W4Params& p, const W4Tile& w, int tid, uint8_t* sc, uint8_t* zp) const {
        const int r = tid >> 2;
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            if (i * 4 >= w.n_groups) break;
            const int gr = i * 4 + (tid & 3);
            if constexpr (MX) {
                sc[r * kPitch + gr] = uint8_t(s[i]);
            } else {
                *reinterpret_cast<uint16_t*>(sc + r * kPitch + 2 * gr) = uint16_t(s[i]);
                zp[r * kZeroPitch + gr] = p.zeros ? uint8_t(z[i]) : uint8_t(8);
            }
        }
    }
};

// STEPS steps of a slot, from i0 on, of NT x 16 rows of the weight (src, 16 rows 2 KB) times MT x 16 rows of x (xb; chunk c
// of row r at slot c ^ (r % 16)), added to sum: lane (g, j) has rows 4 g + e of x and row j of the weight.
// STAGED: x lies in the order of widen's EVEN_ODD, and its sums over the groups were taken before (x_sums, those of the
// lane's rows; otherwise by one more MFMA a step).
template <int DT, bool MX, int XR, int MT, int NT, int STEPS, int GS, bool STAGED>
__device__ __forceinline__ void slot_products(const W4Params& p, const uint8_t* src, const uint8_t* xb, int jx, int i0,
                                              const uint8_t* sc_row, const uint8_t* zp_row, int k0, int gr0, int lane,
                                              const f32x4 (&x_sums)[STEPS / GS], f32x4 (&sum)[NT][MT]) {
    const int g = lane >> 4, j = lane & 15;
    const i32x4 ones = DT == NMM_BF16 ? i32x4{0x3F803F80, 0x3F803F80, 0x3F803F80, 0x3F803F80}
                                      : i32x4{0x3C003C00, 0x3C003C00, 0x3C003C00, 0x3C003C00};
    i32x4 xf[STEPS][MT];
    uint32_t q[STEPS][NT];
    uint32_t sv[NT][STEPS / GS], zv[NT][STEPS / GS];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            q[i][t] = *reinterpret_cast<const uint32_t*>(src + (t * kTileBytes + j * 128 + (((i0 + i) ^ ((j >> 1) & 7)) << 4) + 4 * g));
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            xf[i][mt] = *reinterpret_cast<const i32x4*>(xb + (16 * mt + jx) * 512 + (((4 * (i0 + i) + g) ^ jx) << 4));
        if constexpr (NT > 1) __builtin_amdgcn_sched_barrier(0);      // (as read here: see kTileBytes)
    }
    // (gr0 is a multiple of STEPS / GS: a slice starts with a group, or GS = STEPS)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        read_small<STEPS / GS, Scales<MX, XR>::kSize>(sc_row + 16 * t * Scales<MX, XR>::kPitch + gr0 * Scales<MX, XR>::kSize, sv[t]);
        if constexpr (!MX) read_small<STEPS / GS, 1>(zp_row + 16 * t * Scales<MX, XR>::kZeroPitch + gr0, zv[t]);
    }
    f32x4 acc[NT][MT], xs[MT];
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        if (i % GS == 0) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                xs[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[t][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
        if constexpr (!MX && !STAGED) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) xs[mt] = mfma<DT>(xf[i][mt], ones, xs[mt]);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const i32x4 wf = widen<DT, MX, STAGED>(q[i][t]);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[t][mt] = mfma<DT>(xf[i][mt], wf, acc[t][mt]);
        }
        if (i % GS == GS - 1) {
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                // (a group that starts past K has no scale)
                const float s = k0 + 32 * (i / GS * GS) < p.K ? scale_value<DT, MX>(sv[t][i / GS]) : 0.f;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float xe = STAGED ? x_sums[i / GS][e] : xs[mt][e];
                        const float a = MX ? acc[t][mt][e] : __builtin_fmaf(-float(zv[t][i / GS]), xe, acc[t][mt][e]);
                        sum[t][mt][e] = __builtin_fmaf(s, a, sum[t][mt][e]);
                    }
            }
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (read before the ring is loaded again)
}

// y (the wave has the weight's 16 rows `tile16`), or the slice's part of it and, for the workgroup that comes last, the sum of the parts.
template <int XR, int MT>
__device__ __forceinline__ void finish(const W4Params& p, const W4Tile& w, int tid, int threads, int tile16, const f32x4 (&sum)[MT]) {
    __shared__ int s_last;
    const int lane = tid & 63, g = lane >> 4, col = tile16 * 16 + (lane & 15);
    if (p.ks == 1) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int m = 16 * mt + 4 * g + e, n = w.n0 + col;
                if (m < w.mrows && n < p.N) p.y[int64_t(w.m0 + m) * p.ldy + n] = sum[mt][e];
            }
        return;
    }
    const int64_t tile = int64_t(w.rb) * p.mblocks + w.mb;
    const int part = XR * w.rows;
    const __amdgpu_buffer_rsrc_t pr =
        __builtin_amdgcn_make_buffer_rsrc(p.part + tile * p.ks * part, (short)0, int(uint32_t(p.ks * part) * 4u), kRsrcWord3);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = 16 * mt + 4 * g + e;
            if (m < w.mrows)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(sum[mt][e]), pr,
                                                      uint32_t(w.slice * part + m * w.rows + col) * 4u, 0, kDevice);
        }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0) s_last = arrive(p.tickets + tile, unsigned(p.ks));
    __syncthreads();
    if (!s_last) return;
    // four columns a thread, two of them at once and four slices: one round trip for most
    constexpr int kBatch = 4, kPieces = 2;
    const int total = w.rows * w.mrows;
    for (int o0 = 4 * tid; o0 < total; o0 += 4 * kPieces * threads) {
        f32x4 v[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q0 = 0; q0 < p.ks; q0 += kBatch) {
            f32x4 u[kPieces][kBatch];
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int q = 0; q < kBatch; ++q) {
                    const int o = o0 + 4 * i * threads;
                    u[i][q] = __builtin_bit_cast(
                        f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                   pr, q0 + q < p.ks && o < total ? uint32_t((q0 + q) * part + o) * 4u : kOutOfRange, 0, kDevice));
                }
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
#pragma unroll
                for (int q = 0; q < kBatch; ++q) v[i] += u[i][q];
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int o = o0 + 4 * i * threads;
            const int m = o / w.rows, n = w.n0 + o - m * w.rows;
            if (o >= total) break;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < p.N) p.y[int64_t(w.m0 + m) * p.ldy + n + e] = v[i][e];
        }
    }
}

// Up to 8 rows of x.  XR: rows of x staged (1, 2, 4, 8); GS: steps of a group within a slot (1, 2, 4, or 8 for groups of
// 256 k and more).
template <int DT, bool MX, int XR, int GS>
__global__ __launch_bounds__(64 * kMaxWaves) void w4_few_kernel(const W4Params p) {
    constexpr int D = kFewDepth;
    constexpr int kSlotBytes = 2048;                     // of a wave
    __shared__ __attribute__((aligned(256))) uint8_t xs_buf[XR * kFewSlots * kSlotK * 2];
    __shared__ __attribute__((aligned(128))) uint8_t ring0[kMaxWaves * kSlotBytes];
    __shared__ __attribute__((aligned(128))) uint8_t ring1[kMaxWaves * kSlotBytes];
    __shared__ __attribute__((aligned(128))) uint8_t ring2[kMaxWaves * kSlotBytes];
    __shared__ __attribute__((aligned(128))) uint8_t ring3[kMaxWaves * kSlotBytes];
    static_assert(D == 4, "four rings");
    __shared__ __attribute__((aligned(16))) float x_sum[MX ? 4 : kFewSlots * (kSteps / GS) * XR];
    __shared__ __attribute__((aligned(16))) uint8_t sc[16 * kMaxWaves * Scales<MX, XR>::kPitch];
    __shared__ __attribute__((aligned(16))) uint8_t zp[MX ? 16 : 16 * kMaxWaves * Scales<MX, XR>::kZeroPitch];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    W4Tile w;
    if (!tile_of(p, XR, p.waves, &w)) return;
    const int n_slots = w.slot1 - w.slot0;
    const __amdgpu_buffer_rsrc_t wr = weight_resource(p), xr = x_resource(p, w);
    WaveRows rows;
    rows.init(p, w.n0 + 16 * wave, lane);
    auto load_slot = [&](int sl, uint8_t* ring) {
        const int k0 = (w.slot0 + sl) * kSlotK;
        rows.load(wr, k0, sl < n_slots ? p.K - k0 : 0, ring + wave * kSlotBytes);
    };
    // the scales are loaded first, to registers, then x and the ring's first slots: all of it is in flight at once
    Scales<MX, XR> scales;
    scales.load(p, w, tid);
    // x: half a row's slot (32 chunks of 8 k) in half a load: unit u is slot u / XR of row u % XR
    const int units = XR * n_slots;
    for (int u0 = 2 * wave; u0 < units; u0 += 2 * p.waves) {
        const int u = u0 + (lane >> 5);
        const int r = u & (XR - 1), sl = u / XR;
        const int k = (w.slot0 + sl) * kSlotK + 8 * ((lane & 31) ^ r);
        const uint32_t o = u < units && r < w.mrows && k < p.K ? uint32_t((int64_t(r) * p.ldx + k) * 2) : kOutOfRange;
        load_x(xr, o, xs_buf + u0 * 512);
    }
    load_slot(0, ring0);
    load_slot(1, ring1);
    load_slot(2, ring2);
    load_slot(3, ring3);
    scales.store(p, w, tid, sc, zp);
    // (x has landed once at most the weight's loads are outstanding; those stay in flight)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * D) : "memory");
    // What a chunk that K ends in holds past K is cleared; beside zero points, the chunks are put into widen's order and
    // their sums taken, 4 GS chunks a group.
    constexpr int kGroups = kSteps / GS;                 // groups of a slot
    if (!MX || p.K % 8) {
        for (int c = tid; c < XR * n_slots * 32; c += 64 * p.waves) {
            const int u = c >> 5, r = u & (XR - 1), sl = u / XR;
            i32x4* const at = reinterpret_cast<i32x4*>(xs_buf + u * 512 + (((c & 31) ^ r) << 4));
            i32x4 v = *at;
            const int left = p.K - ((w.slot0 + sl) * kSlotK + 8 * (c & 31));
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = left > 2 * e + 1 ? v[e] : left > 2 * e ? v[e] & 0xFFFF : 0;
            }
            if constexpr (!MX) {
                float t = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) t += value<DT>(uint32_t(v[e]) & 0xFFFFu) + value<DT>(uint32_t(v[e]) >> 16);
                t += dpp<0xB1>(t);                                   // lane ^ 1
                t += dpp<0x4E>(t);                                   // lane ^ 2
                if constexpr (GS > 1) t += dpp<0x141>(t);            // the mirrored lane of 8
                if constexpr (GS > 2) t += dpp<0x140>(t);            // of 16
                if constexpr (GS > 4) t += __shfl_xor(t, 16);
                if ((c & (4 * GS - 1)) == 0) x_sum[(sl * kGroups + (c & 31) / (4 * GS)) * XR + r] = t;
                v = i32x4{int(__builtin_amdgcn_perm(v[1], v[0], 0x05040100u)), int(__builtin_amdgcn_perm(v[3], v[2], 0x05040100u)),
                          int(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u)), int(__builtin_amdgcn_perm(v[3], v[2], 0x07060302u))};
            }
            *at = v;
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }

    f32x4 sum[1][1] = {{f32x4{0.f, 0.f, 0.f, 0.f}}};
    const int jx = lane & (XR - 1);
    const int row = 16 * wave + (lane & 15);
    auto consume = [&](const uint8_t* ring, int sl) {
        // the slot has landed once at most the younger slots' loads are outstanding (loads complete in order)
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * (D - 1)) : "memory");
        const int k0 = (w.slot0 + sl) * kSlotK;
        // rows 4 g + e of x, of XR
        f32x4 x_sums[kGroups];
        if constexpr (!MX) {
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const float* const t = x_sum + (sl * kGroups + i) * XR + (XR == 8 ? 4 * ((lane >> 4) & 1) : 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) x_sums[i][e] = t[e & (XR - 1)];
            }
        }
        slot_products<DT, MX, XR, 1, 1, kSteps, GS, true>(
            p, ring + wave * kSlotBytes, xs_buf + sl * XR * 512, jx, 0, sc + row * Scales<MX, XR>::kPitch,
            zp + (MX ? 0 : row * Scales<MX, XR>::kZeroPitch), k0, (k0 >> p.lg_group) - w.group0, lane, x_sums, sum);
    };
    for (int sl = 0; sl < n_slots; sl += D) {
        consume(ring0, sl);
        load_slot(sl + D, ring0);
        if (sl + 1 < n_slots) consume(ring1, sl + 1);
        load_slot(sl + D + 1, ring1);
        if (sl + 2 < n_slots) consume(ring2, sl + 2);
        load_slot(sl + D + 2, ring2);
        if (sl + 3 < n_slots) consume(ring3, sl + 3);
        load_slot(sl + D + 3, ring3);
    }
    __builtin_amdgcn_s_waitcnt(0);        // (no load may write LDS after the workgroup has left)
    finish<XR, 1>(p, w, tid, 64 * p.waves, wave, sum[0]);
}

// More rows of x: XR = 16 MT of them, a slot of which lies in the ring beside the weight's, shared by the 8 waves: wave
// w multiplies 32 rows of the weight, w % 4, and half of a slot's steps, w / 4.
template <int DT, bool MX, int MT, int GS>
__global__ __launch_bounds__(64 * kMaxWaves) void w4_rows_kernel(const W4Params p) {
    constexpr int XR = 16 * MT, D = kRowsDepth;
    constexpr int kWeightBytes = kMaxWaves * kTileBytes, kRingBytes = kWeightBytes + XR * 512;
    constexpr int kLoads = 2 + MT;                       // of a wave, a slot
    __shared__ __attribute__((aligned(256))) uint8_t ring0[kRingBytes];
    __shared__ __attribute__((aligned(256))) uint8_t ring1[kRingBytes];
    __shared__ __attribute__((aligned(256))) uint8_t ring2[kRingBytes];
    __shared__ __attribute__((aligned(256))) uint8_t ring3[kRingBytes];
    static_assert(D == 4, "four rings");
    __shared__ __attribute__((aligned(16))) uint8_t sc[16 * kMaxWaves * Scales<MX, XR>::kPitch];
    __shared__ __attribute__((aligned(16))) uint8_t zp[MX ? 16 : 16 * kMaxWaves * Scales<MX, XR>::kZeroPitch];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    W4Tile w;
    if (!tile_of(p, XR, kMaxWaves, &w)) return;
    const int n_slots = w.slot1 - w.slot0;
    const __amdgpu_buffer_rsrc_t wr = weight_resource(p), xr = x_resource(p, w);
    WaveRows rows;
    rows.init(p, w.n0 + 16 * wave, lane);
    // x: two rows' slots a load
    uint32_t xoff[MT];
    int xk[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int r = 2 * (wave * MT + i) + (lane >> 5);
        xk[i] = 8 * ((lane & 31) ^ (r & 15));
        xoff[i] = r < w.mrows ? uint32_t((int64_t(r) * p.ldx + xk[i]) * 2) : kOutOfRange;
    }
    auto load_slot = [&](int sl, uint8_t* ring) {
        const int k0 = (w.slot0 + sl) * kSlotK;
        const int left = sl < n_slots ? p.K - k0 : 0;
        rows.load(wr, k0, left, ring + wave * kTileBytes);
#pragma unroll
        for (int i = 0; i < MT; ++i)
            load_x(xr, xk[i] < left ? xoff[i] + uint32_t(k0) * 2u : kOutOfRange,
                   ring + kWeightBytes + (wave * MT + i) * 1024);
    };
    Scales<MX, XR> scales;
    scales.load(p, w, tid);
    load_slot(0, ring0);
    load_slot(1, ring1);
    load_slot(2, ring2);
    scales.store(p, w, tid, sc, zp);

    constexpr int kHalf = kSteps / 2, kGS = GS < kHalf ? GS : kHalf;
    const int pair = wave & 3, half = wave >> 2;
    f32x4 sum[2][MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) sum[0][mt] = sum[1][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int row = 32 * pair + (lane & 15);
    // the slot has landed, for every wave, and every wave has read the slot before, whose ring is loaded again
    auto step = [&](uint8_t* ring, uint8_t* before, int sl) {
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((D - 2) * kLoads) : "memory");
        load_slot(sl + D - 1, before);
        const int k0 = (w.slot0 + sl) * kSlotK;
        // what a chunk that K ends in holds past K is cleared
        if (p.K % 8 && p.K - k0 < kSlotK && p.K > k0) {
            const int c = (p.K - k0) / 8;
            if (tid < XR * 8 && tid % 8 >= p.K % 8) {
                const int r = tid / 8;
                *reinterpret_cast<uint16_t*>(ring + kWeightBytes + r * 512 + ((c ^ (r & 15)) << 4) + 2 * (tid % 8)) = 0;
            }
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        }
        f32x4 none[kHalf / kGS];
        const int kh = k0 + half * kHalf * 32;
        slot_products<DT, MX, XR, MT, 2, kHalf, kGS, false>(
            p, ring + pair * 2 * kTileBytes, ring + kWeightBytes, lane & 15, half * kHalf, sc + row * Scales<MX, XR>::kPitch,
            zp + (MX ? 0 : row * Scales<MX, XR>::kZeroPitch), kh, (kh >> p.lg_group) - w.group0, lane, none, sum);
    };
    for (int sl = 0; sl < n_slots; sl += D) {
        step(ring0, ring3, sl);
        if (sl + 1 >= n_slots) break;
        step(ring1, ring0, sl + 1);
        if (sl + 2 >= n_slots) break;
        step(ring2, ring1, sl + 2);
        if (sl + 3 >= n_slots) break;
        step(ring3, ring2, sl + 3);
    }
    __builtin_amdgcn_s_waitcnt(0);        // (no load may write LDS after the workgroup has left)
    // each wave of a pair hands the other half's sums of one tile over and keeps the other tile
    __syncthreads();
    f32x4* const xchg = reinterpret_cast<f32x4*>(ring0);                   // [wave][MT][lane]
    f32x4 mine[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        mine[mt] = half ? sum[1][mt] : sum[0][mt];
        xchg[(wave * MT + mt) * 64 + lane] = half ? sum[0][mt] : sum[1][mt];
    }
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const f32x4 other = xchg[((wave ^ 4) * MT + mt) * 64 + lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[mt][e] += other[e];
    }
    finish<XR, MT>(p, w, tid, 64 * kMaxWaves, 2 * pair + half, mine);
}

// ---------------------------------------------------------------------------------------------
// The partition.
// ---------------------------------------------------------------------------------------------
struct W4Plan {
    int xr = 1, waves = 4;
    int row_blocks = 1, mblocks = 1, ks = 1, slots = 1, slots_per_slice = 1;
    int64_t grid = 0;
    size_t ws_bytes = 0;
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t kLim = int64_t(1) << 31;
// The partition's estimate, in the time that a wave's slot of 2 KB takes at a CU's share of the memory rate (170 cycles): a CU
// takes its workgroups one after the other, each its waves' slots and a start (2 us), and a split K once the hand-over
// (1.4 us).  One row, K 16384, N 7168: 16.5 us in 256 workgroups of 7 waves and 16 slots; in workgroups of 4 waves, two a
// CU, 17.8 in 448 and 21.5 in 560, which are 3 on some CUs; K 512, N 512: 4.2 us in 8 workgroups of 4 waves, 4.7 in 4 of 8.
constexpr int64_t kCus = 256;
constexpr int64_t kStartCost = 28, kSplitCost = 20;

nmm_status plan_w4(int64_t M, int64_t K, int64_t N, bool mx, int64_t group, W4Plan* out) {
    W4Plan q;
    if (M <= 0 || K <= 0 || N <= 0) {
        *out = q;
        return NMM_OK;
    }
    q.xr = M <= 1 ? 1 : M <= 2 ? 2 : M <= 4 ? 4 : M <= 8 ? 8 : M <= 16 ? 16 : 32;
    q.mblocks = static_cast<int>(cdiv(M, q.xr));
    q.slots = static_cast<int>(cdiv(K, kSlotK));
    const bool few = q.xr <= kFewRows;
    const int64_t most = std::min<int64_t>(few ? kFewSlots : 64, std::max<int64_t>(1, max_groups(mx, q.xr) * group / kSlotK));
    int64_t best = INT64_MAX;
    for (int waves = kMaxWaves; waves >= (few ? 4 : kMaxWaves); --waves) {
        const int64_t tiles = cdiv(N, 16 * waves) * q.mblocks;
        for (int64_t per = std::min<int64_t>(most, q.slots); per >= 1; --per) {
            const int64_t ks = cdiv(q.slots, per);
            if (ks > 1 && tiles > kMaxTickets) break;
            const int64_t cost = cdiv(tiles * ks, kCus) * (per * waves + kStartCost) + (ks > 1 ? kSplitCost : 0);
            if (cost >= best) continue;
            best = cost;
            q.waves = waves;
            q.row_blocks = static_cast<int>(cdiv(N, 16 * waves));
            q.ks = static_cast<int>(ks);
            q.slots_per_slice = static_cast<int>(per);
        }
    }
    if (best == INT64_MAX) return NMM_ERR_SHAPE;
    q.grid = cdiv(q.row_blocks, 8) * 8 * q.mblocks * q.ks;
    if (q.grid >= (int64_t(1) << 32) / (64 * kMaxWaves)) return NMM_ERR_SHAPE;
    if (q.ks > 1)
        q.ws_bytes = size_t(kTicketBytes) + size_t(q.row_blocks) * q.mblocks * q.ks * q.xr * 16 * q.waves * 4;
    *out = q;
    return NMM_OK;
}

// Rows of x per launch: more row blocks than there are tickets (handoff.h) are split over launches, which follow each other on
// the stream and may use one workspace.  (N of 2^21 and more has K < 2048 and is never split.)
int64_t launch_rows(int64_t M, int64_t N) {
    return std::min<int64_t>(M, kMaxRows * std::max<int64_t>(1, kMaxTickets / cdiv(N, 16 * kMaxWaves)));
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int DT, bool MX, int GS>
void launch_xr(const W4Params& p, const W4Plan& q, hipStream_t s) {
    const dim3 grid(static_cast<uint32_t>(q.grid)), block(64 * q.waves);
    switch (q.xr) {
        case 1: hipLaunchKernelGGL((w4_few_kernel<DT, MX, 1, GS>), grid, block, 0, s, p); break;
        case 2: hipLaunchKernelGGL((w4_few_kernel<DT, MX, 2, GS>), grid, block, 0, s, p); break;
        case 4: hipLaunchKernelGGL((w4_few_kernel<DT, MX, 4, GS>), grid, block, 0, s, p); break;
        case 8: hipLaunchKernelGGL((w4_few_kernel<DT, MX, 8, GS>), grid, block, 0, s, p); break;
        case 16: hipLaunchKernelGGL((w4_rows_kernel<DT, MX, 1, GS>), grid, block, 0, s, p); break;
        default: hipLaunchKernelGGL((w4_rows_kernel<DT, MX, 2, GS>), grid, block, 0, s, p); break;
    }
}

template <int DT>
void launch(const W4Params& p, const W4Plan& q, bool mx, hipStream_t s) {
    if (mx) return launch_xr<DT, true, 1>(p, q, s);
    switch (p.lg_group) {
        case 5: return launch_xr<DT, false, 1>(p, q, s);
        case 6: return launch_xr<DT, false, 2>(p, q, s);
        case 7: return launch_xr<DT, false, 4>(p, q, s);
        default: return launch_xr<DT, false, 8>(p, q, s);
    }
}

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_gemv_w4_workspace_size(int64_t M, int64_t K, int64_t N, int64_t group) {
    if (M <= 0 || K <= 0 || N <= 0 || M >= kLim || K >= kLim || N >= kLim || group < 32 || (group & (group - 1))) return 0;
    const int64_t step = launch_rows(M, N);
    size_t most = 0;
    for (const bool mx : {false, true}) {
        if (mx && group != 32) continue;
        for (const int64_t rows : {step, M % step ? M % step : step}) {
            W4Plan q;
            if (plan_w4(rows, K, N, mx, group, &q) != NMM_OK) return 0;
            most = std::max(most, q.ws_bytes);
        }
    }
    return most;
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
    const int64_t step = launch_rows(M, N);
    W4Plan first, last;
    const bool mx = format == NMM_W4_MX;
    nmm_status st = plan_w4(step, K, N, mx, group, &first);
    if (st == NMM_OK) st = plan_w4(M % step ? M % step : step, K, N, mx, group, &last);
    if (st != NMM_OK) return st;
    st = validate_workspace(workspace, workspace_bytes, std::max(first.ws_bytes, last.ws_bytes));
    if (st != NMM_OK) return st;
    W4Params p{};
    p.ldx = ldx;
    p.w = static_cast<const uint8_t*>(Wq);
    p.scales = static_cast<const uint8_t*>(scales);
    p.zeros = zeros;
    p.lds = lds;
    p.ldz = ldz;
    p.ldy = ldy;
    if (workspace) {
        p.tickets = static_cast<unsigned*>(workspace);
        p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
    }
    p.row_bytes = static_cast<uint32_t>(ldwq);
    p.w_extent = static_cast<uint32_t>(w_extent);
    p.K = static_cast<int>(K);
    p.N = static_cast<int>(N);
    p.groups = static_cast<int>(groups);
    while ((int64_t(1) << p.lg_group) < group) ++p.lg_group;
    for (int64_t m = 0; m < M; m += step) {
        const W4Plan& q = M - m >= step ? first : last;
        p.x = static_cast<const uint16_t*>(x) + m * ldx;
        p.y = y + m * ldy;
        p.M = static_cast<int>(std::min(step, M - m));
        p.row_blocks = q.row_blocks;
        p.mblocks = q.mblocks;
        p.ks = q.ks;
        p.slots_per_slice = q.slots_per_slice;
        p.slots = q.slots;
        p.waves = q.waves;
        if (dt == NMM_BF16) launch<NMM_BF16>(p, q, mx, static_cast<hipStream_t>(stream));
        else launch<NMM_F16>(p, q, mx, static_cast<hipStream_t>(stream));
    }
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
