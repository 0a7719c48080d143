// What the kernels over weights given as [N, K] share: the ring of a wave in LDS, filled by LDS-direct loads of 4 rows x 256
// bytes, and the fragments of v_mfma_f32_16x16x32 read from it (the reasons stand in mfma_nt.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "nmm_internal.h"

namespace nmm {
namespace ring {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kRsrcWord3 = 0x00020000;
constexpr int kLoadNT = 2;
constexpr uint32_t kOutOfRange = 0x80000000u;
constexpr int kRowBytes = kMfmaNtGroup * 2;     // bytes of one row in a group: 16 chunks
constexpr int kQuad = 4 * kRowBytes;            // one LDS-direct load: 4 rows of a group

template <int DT>
__device__ __forceinline__ f32x4 mfma(i32x4 a, i32x4 b, f32x4 c) {
    if constexpr (DT == NMM_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The first `left` of a chunk's 8 values, zeros after them.
__device__ __forceinline__ i32x4 keep_first(i32x4 v, int left) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] &= (2 * e + 1 < left) ? -1 : (2 * e < left ? 0x0000FFFF : 0);
    return v;
}

// The fragments of two MFMA steps from LDS: once at most VM of the wave's loads are outstanding, F
// fragments at addresses a and b each (fragment f at byte offset OFF + 4096 f, the x fragments of the
// last MT at XOFF + 4096 f from ax and bx), complete when this returns.  The loads that fill LDS are
// LDS-direct: the compiler would wait for all of them before any read that may alias, so the wait
// and the reads are written out.
template <int VM, int NT, int MT, int OFF, int XOFF>
__device__ __forceinline__ void read_pair(i32x4 (&w0)[NT], i32x4 (&w1)[NT], i32x4 (&x0)[MT], i32x4 (&x1)[MT], uint32_t a,
                                          uint32_t b, uint32_t ax, uint32_t bx) {
    static_assert(VM < 64 && OFF + 4096 * NT < 65536 && XOFF + 4096 * MT < 65536, "immediate fields");
    if constexpr (NT == 1 && MT == 1)
        asm volatile("s_waitcnt vmcnt(%8)\n\tds_read_b128 %0, %4 offset:%9\n\tds_read_b128 %1, %5 offset:%9\n\t"
                     "ds_read_b128 %2, %6 offset:%10\n\tds_read_b128 %3, %7 offset:%10\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w0[0]), "=&v"(w1[0]), "=&v"(x0[0]), "=&v"(x1[0])
                     : "v"(a), "v"(b), "v"(ax), "v"(bx), "n"(VM), "n"(OFF), "n"(XOFF) : "memory");
    else if constexpr (NT == 2 && MT == 1)
        asm volatile("s_waitcnt vmcnt(%10)\n\tds_read_b128 %0, %6 offset:%11\n\tds_read_b128 %1, %7 offset:%11\n\t"
                     "ds_read_b128 %2, %6 offset:%12\n\tds_read_b128 %3, %7 offset:%12\n\t"
                     "ds_read_b128 %4, %8 offset:%13\n\tds_read_b128 %5, %9 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w0[0]), "=&v"(w1[0]), "=&v"(w0[1]), "=&v"(w1[1]), "=&v"(x0[0]), "=&v"(x1[0])
                     : "v"(a), "v"(b), "v"(ax), "v"(bx), "n"(VM), "n"(OFF), "n"(OFF + 4096), "n"(XOFF) : "memory");
    else if constexpr (NT == 1 && MT == 2)
        asm volatile("s_waitcnt vmcnt(%10)\n\tds_read_b128 %0, %6 offset:%11\n\tds_read_b128 %1, %7 offset:%11\n\t"
                     "ds_read_b128 %2, %8 offset:%12\n\tds_read_b128 %3, %9 offset:%12\n\t"
                     "ds_read_b128 %4, %8 offset:%13\n\tds_read_b128 %5, %9 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w0[0]), "=&v"(w1[0]), "=&v"(x0[0]), "=&v"(x1[0]), "=&v"(x0[1]), "=&v"(x1[1])
                     : "v"(a), "v"(b), "v"(ax), "v"(bx), "n"(VM), "n"(OFF), "n"(XOFF), "n"(XOFF + 4096) : "memory");
    else
        asm volatile("s_waitcnt vmcnt(%12)\n\tds_read_b128 %0, %8 offset:%13\n\tds_read_b128 %1, %9 offset:%13\n\t"
                     "ds_read_b128 %2, %8 offset:%14\n\tds_read_b128 %3, %9 offset:%14\n\t"
                     "ds_read_b128 %4, %10 offset:%15\n\tds_read_b128 %5, %11 offset:%15\n\t"
                     "ds_read_b128 %6, %10 offset:%16\n\tds_read_b128 %7, %11 offset:%16\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w0[0]), "=&v"(w1[0]), "=&v"(w0[1]), "=&v"(w1[1]), "=&v"(x0[0]), "=&v"(x1[0]), "=&v"(x0[1]), "=&v"(x1[1])
                     : "v"(a), "v"(b), "v"(ax), "v"(bx), "n"(VM), "n"(OFF), "n"(OFF + 4096), "n"(XOFF), "n"(XOFF + 4096) : "memory");
}

}  // namespace ring
}  // namespace nmm
