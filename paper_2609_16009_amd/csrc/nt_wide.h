// The products of nt_rows.h for many rows of x a tile (device code).
//
// A workgroup of 8 waves owns a tile of BM rows of x and BN rows of the weight.  Slots of 64 k of both lie in a ring of S in
// LDS, filled by LDS-direct loads of 8 rows x 128 bytes, S - 1 slots ahead, with one barrier a slot; a wave multiplies its
// part of the tile with v_mfma_f32_16x16x32.  Chunk c of row r sits at place c ^ (r / 2 % 8) of its 128 bytes: LDS serves 256
// bytes a cycle, the 16 rows of a fragment's quarter wave, which then lie in 16 different places.
// The weight is the A operand and x the B operand: a lane ends with four consecutive n of one m.  Where a gate
// multiplies, a wave's rows of the weight are half the gate's and half those that they are multiplied with.
// Two waves a SIMD, so that one reads fragments while the other's are multiplied: the reads wait for themselves (see
// read_tiles), as the compiler makes a read of LDS wait for loads into other slots too.
#pragma once

#include "nt_rows.h"

namespace nmm {
namespace rows {

constexpr int kWideWaves = 8;
constexpr int kWideThreads = 64 * kWideWaves;
constexpr int kWideK = 64;                      // k of a slot
constexpr int kWideRow = 2 * kWideK;            // bytes of a row in a slot
constexpr int kWideTile = 16 * kWideRow;        // and of 16 rows

template <int N>
__device__ __forceinline__ void wait_loads() {
    static_assert(N >= 0 && N < 64, "vmcnt holds 6 bits");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// The fragments of two tiles of the weight (at wa and kWideTile behind it) and of MT tiles of x, complete when this returns.
template <int MT>
__device__ __forceinline__ void read_tiles(i32x4 (&w)[2], i32x4 (&x)[MT], uint32_t wa, uint32_t xa) {
    static_assert(MT == 1 || MT == 2 || MT == 4, "tiles of x");
    if constexpr (MT == 1)
        asm volatile("ds_read_b128 %0, %3\n\tds_read_b128 %2, %4\n\tds_read_b128 %1, %3 offset:%5\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w[0]), "=&v"(w[1]), "=&v"(x[0]) : "v"(wa), "v"(xa), "n"(kWideTile) : "memory");
    else if constexpr (MT == 2)
        asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %2, %5\n\tds_read_b128 %1, %4 offset:%6\n\t"
                     "ds_read_b128 %3, %5 offset:%6\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(w[0]), "=&v"(w[1]), "=&v"(x[0]), "=&v"(x[1]) : "v"(wa), "v"(xa), "n"(kWideTile) : "memory");
    else
        asm volatile("ds_read_b128 %0, %6\n\tds_read_b128 %2, %7\n\tds_read_b128 %1, %6 offset:%8\n\t"
                     "ds_read_b128 %3, %7 offset:%8\n\tds_read_b128 %4, %7 offset:%9\n\tds_read_b128 %5, %7 offset:%10\n\t"
                     "s_waitcnt lgkmcnt(0)"
                     : "=&v"(w[0]), "=&v"(w[1]), "=&v"(x[0]), "=&v"(x[1]), "=&v"(x[2]), "=&v"(x[3])
                     : "v"(wa), "v"(xa), "n"(kWideTile), "n"(2 * kWideTile), "n"(3 * kWideTile) : "memory");
}

template <int DT, int MODE, int BM, int BN, int S>
__global__ __launch_bounds__(kWideThreads) void wide_kernel(const RowsParams p) {
    constexpr int NT = 2, WN = BN / 16 / NT, WM = kWideWaves / WN;       // waves along n and m; a wave's 16-row tiles
    constexpr int MT = BM / WM / 16;
    constexpr int kLoads = (BM + BN) / 8 / kWideWaves;                   // loads of a slot per wave
    constexpr int kSlot = (BM + BN) * kWideRow;
    static_assert(WM * WN == kWideWaves && MT * WM * 16 == BM && kLoads * 8 * kWideWaves == BM + BN && BN % 64 == 0 && S >= 3,
                  "whole tiles and loads a wave");
    __shared__ __attribute__((aligned(256))) uint8_t ring[S * kSlot];
    __shared__ int starts[MODE == kDense ? 1 : kMaxExperts + 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, j = lane & 15;
    const int wm = wave % WM, wn = wave / WM;
    const bool gated = MODE == kUp || (MODE == kDense && p.gated);
    const int n_step = gated ? BN / 2 : BN;

    if constexpr (MODE != kDense) scan_tiles<BM, kWideThreads>(p, starts);
    const int64_t nb8 = (p.n_blocks + 7) >> 3;
    const int64_t total = (MODE == kDense ? (int64_t(p.M) + BM - 1) / BM : int64_t(__builtin_amdgcn_readfirstlane(starts[p.local]))) * nb8;
    const int steps = (p.K + kWideK - 1) / kWideK;
    // the lane's chunk of a load: the same of every load of its wave (they are 64 rows apart)
    const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
    // fragments: row j of a tile, chunk g; chunk 4 + g lies 64 bytes away
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((lds_void*)ring)) + j * kWideRow + ((g ^ (j >> 1)) << 4);
    const uint32_t wa = base + wn * NT * kWideTile, xa = base + BN * kWideRow + wm * MT * kWideTile;

    for (int64_t idx = blockIdx.x >> 3; idx < total; idx += gridDim.x >> 3) {
        Item it;
        if (!item_of<MODE, BM>(p, starts, idx, blockIdx.x & 7, &it)) continue;
        const int n0 = it.nb * n_step;
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(p.w + it.e * p.w_stride), (short)0, (int)p.w_extent, kRsrcWord3);
        const uint16_t* xb = p.x;
        uint32_t x_extent = p.x_extent;
        if constexpr (MODE != kUp) {
            xb += (int64_t(it.first) + it.m0) * p.ldx;
            x_extent = uint32_t((int64_t(it.mrows - 1) * p.ldx + (p.K + 7) / 8 * 8) * 2);
        }
        const __amdgpu_buffer_rsrc_t xr =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(xb), (short)0, (int)x_extent, kRsrcWord3);
        uint32_t off[kLoads];      // byte offset of the lane's chunk in slot 0; out of range where there is none
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = 8 * (wave + kWideWaves * i) + (lane >> 3);
            if (64 * i < BN) {     // (a row of the weight for every wave)
                constexpr int kWaveRows = BN / WN;
                int64_t row = n0 + r;
                bool ok = row < p.N;
                if (gated) {
                    const int rr = r % kWaveRows, n = n0 + r / kWaveRows * (kWaveRows / 2) + rr % (kWaveRows / 2);
                    ok = n < p.N;
                    row = rr < kWaveRows / 2 ? n : int64_t(p.N) + n;
                }
                off[i] = ok ? uint32_t(row * p.row_bytes) + 16u * chunk : kOutOfRange;
            } else {
                const int m = r - BN;
                bool ok = m < it.mrows;
                int64_t row = m;
                if constexpr (MODE == kUp) {
                    const int pair = ok ? p.pairs[it.first + it.m0 + m] : -1;
                    ok = uint32_t(pair) < uint32_t(p.M);
                    row = pair / p.top_k;
                }
                off[i] = ok ? uint32_t(row * p.ldx * 2) + 16u * chunk : kOutOfRange;
            }
        }
        auto load_slot = [&](int step, int slot) {
            const int kg = step * kWideK;
            // past K out of range, which the top bit says (extents are below 2^31)
            const uint32_t past = kg + 8 * chunk < p.K ? 0u : kOutOfRange;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t o = (off[i] + uint32_t(kg) * 2u) | past;
                uint8_t* const dst = ring + slot * kSlot + 8 * (wave + kWideWaves * i) * kWideRow;
                if (64 * i < BN) __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)dst, 16, o, 0, 0, 0);
                else __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)dst, 16, o, 0, 0, 0);
            }
        };
        f32x4 sum[NT][MT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};

        // (the loads counted below are the ring's alone; its slots are free)
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < S - 1; ++s) load_slot(s, s);
        int slot = 0;
        for (int step = 0; step < steps; ++step) {
            // this wave's loads of the slot have landed, then every wave's; all are done with the slot that is filled next
            wait_loads<(S - 2) * kLoads>();
            asm volatile("s_barrier" ::: "memory");
            load_slot(step + S - 1, slot == 0 ? S - 1 : slot - 1);
            const bool ragged = (step + 1) * kWideK > p.K && (p.K & 7);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                i32x4 w[NT], x[MT];
                read_tiles<MT>(w, x, (wa ^ (64u * h)) + slot * kSlot, (xa ^ (64u * h)) + slot * kSlot);
                if (ragged) {      // clear what lies past K
                    const int left = p.K - (step * kWideK + 32 * h + 8 * g);
#pragma unroll
                    for (int t = 0; t < NT; ++t) w[t] = keep_first(w[t], left);
#pragma unroll
                    for (int m = 0; m < MT; ++m) x[m] = keep_first(x[m], left);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int m = 0; m < MT; ++m) sum[t][m] = mfma<DT>(w[t], x[m], sum[t][m]);
            }
            slot = slot == S - 1 ? 0 : slot + 1;
        }

#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const int mr = (wm * MT + m) * 16 + j;
            if (mr >= it.mrows) continue;
            int64_t row = int64_t(it.first) + it.m0 + mr;
            if constexpr (MODE == kDown) {
                const int pair = p.pairs[row];
                if (uint32_t(pair) >= uint32_t(p.M)) continue;
                row = pair;
            }
            auto finish = [&](int t, int n) {
                float z[4], z2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = sum[t][m][i];
                if (gated) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) z2[i] = sum[t % (NT / 2) + NT / 2][m][i];
                }
                if (n < p.N) finish4<DT, MODE>(p, row, n, z, z2);
            };
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if (gated) {
                    if (t < NT / 2) finish(t, n0 + (wn * (NT / 2) + t) * 16 + 4 * g);
                } else {
                    finish(t, n0 + (wn * NT + t) * 16 + 4 * g);
                }
            }
        }
    }
    __builtin_amdgcn_s_waitcnt(0);       // the ring's last loads into LDS have landed
}

}  // namespace rows
}  // namespace nmm
