// The products of nt_rows.h for many rows of x a tile (device code).
//
// A workgroup of 8 waves owns a tile of up to BM rows of x and BN rows of the weight.  Slots of 64 k of both lie in a ring of S in
// LDS, filled by LDS-direct loads of 8 rows x 128 bytes, up to S slots ahead; a wave multiplies its part of the tile with
// v_mfma_f32_16x16x32.  Chunk c of row r sits at place c ^ (r / 2 % 8) of its 128 bytes, so that the 16 rows of a fragment's
// quarter wave lie in 16 different places (no bank conflict counted).
// The weight is the A operand and x the B operand: a lane ends with four consecutive n of one m.  Where a gate
// multiplies, a wave's rows of the weight are half the gate's and half those that they are multiplied with.  The 16-row tiles of x are
// dealt to the waves in turn, so that a tile with fewer rows than BM costs what its own rows do.
//
// Reading fragments (about 110 bytes a cycle and CU) takes as long as multiplying them, so the two run beside each other: while one
// half of a slot is multiplied the next one's fragments are read, and the one barrier a slot lies between the halves.  The
// loads are written as asm: the compiler makes a read of LDS wait for every LDS-direct load that it knows of.
//
// What bounds it: how fast a CU is given lines that its L2 does not hold, 25 to 50 GB/s whether 64 or 128 KB of loads are in flight, so
// the weight's bytes and all 256 CUs streaming them.  16 experts of 128 rows on average, 2 x 2048 x 7168: 225 us for 0.94 GB of weights
// (the loads alone 210, reads and products without loads 169); K in four slices for 256 rows of 2 x 2048 x 7168, 21.4 us, of which
// 13 to 14 are the walk over 28 slots (the slope over K), 2 to 3 its sums to memory (21.4 and 19.0 to 19.4 without their stores) and the rest the start
// and the end.  Sums are fp32 in the matrix cores, one chain over K or a slice: relative 2-norm error 8.2e-7 at K = 16384 whole.  Where results are
// asked for in fp32 (F64), chains of four matrix instructions are taken into fp64 every other slot: 6.5e-8 to 7.7e-8 (fp16 9.1e-8) and 29.5 instead of 25.9 us
// for 256 rows of 2 x 2048 x 7168, 76 instead of 63 for 1024 of 4096 x 7168 (every fourth slot: 9.8e-8, 1.2e-7, 28.1 and 71).
#pragma once

#include "nt_rows.h"

namespace nmm {
namespace rows {

constexpr int kWideWaves = 8;
constexpr int kWideThreads = 64 * kWideWaves;
constexpr int kWideK = 64;                      // k of a slot
constexpr int kWideRow = 2 * kWideK;            // bytes of a row in a slot
constexpr int kWideTile = 16 * kWideRow;        // and of 16 rows

// At most N of this wave's loads are outstanding, none of its LDS reads; then every wave's.
template <int N>
__device__ __forceinline__ void slot_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt holds 6 bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// 64 lanes x 16 bytes to LDS from `lds` on (the same in all lanes), lane l's behind lane l - 1's, from byte `offset` of the buffer.
// Not said to touch memory, so that reads of other slots may move past it: what orders it is slot_barrier.
// (m0 is reserved: nothing else in these kernels holds a value in it.  The wait is what a load needs behind a vector instruction that
// wrote its descriptor, which the compiler does not see to inside asm.)
__device__ __forceinline__ void load_to_lds(i32x4 rsrc, uint32_t lds, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(lds), "v"(offset), "s"(rsrc));
}

// The buffer resource as its four words (address, no stride, extent, raw).
__device__ __forceinline__ i32x4 rsrc_words(const void* base, uint32_t extent) {
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    i32x4 r{int(uint32_t(a)), int(uint32_t(a >> 32) & 0xFFFFu), int(extent), kRsrcWord3};
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = __builtin_amdgcn_readfirstlane(r[i]);
    return r;
}

template <int DT, int MODE, int BM, int BN, int S, bool F64 = false>
__global__ __launch_bounds__(kWideThreads) void wide_kernel(const RowsParams p) {
    constexpr int NT = BM >= 256 ? 4 : 2, WN = BN / 16 / NT, WM = kWideWaves / WN;   // a wave's tiles; waves along n and m
    constexpr int MT = BM / WM / 16;
    constexpr int LW = BN / 64, kLoads = LW + BM / 64;                   // loads of a slot per wave, the weight's first
    constexpr int kSlot = (BM + BN) * kWideRow;
    static_assert((MT == 2 || MT == 4) && MT * WM * 16 == BM && NT * WN * 16 == BN && NT % 2 == 0 && S >= 3, "whole tiles, gate and up");
    constexpr int kPitch = BN + 4;                                       // floats of a row of sums
    static_assert(BM * kPitch * 4 <= S * kSlot, "the sums fit the ring");
    __shared__ __attribute__((aligned(256))) uint8_t ring[S * kSlot];
    __shared__ int starts[MODE == kDense ? 1 : kMaxExperts + 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, j = lane & 15;
    const int wm = wave % WM, wn = wave / WM;
    const bool gated = MODE == kUp || (MODE == kDense && p.gated);
    const int n_step = gated ? BN / 2 : BN;

    if constexpr (MODE != kDense) scan_tiles<BM, kWideThreads>(p, starts);
    const int64_t nb8 = blocks_of(p);
    const int64_t total = (MODE == kDense ? (int64_t(p.M) + BM - 1) / BM : int64_t(__builtin_amdgcn_readfirstlane(starts[p.local]))) * nb8;
    const int all_steps = (p.K + kWideK - 1) / kWideK;
    // the lane's chunk of a load: the same of every load of its wave (they are 64 rows apart)
    const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
    // fragments: row j of a tile, chunk g; chunk 4 + g lies 64 bytes away
    const int f0 = j * kWideRow + ((g ^ (j >> 1)) << 4);
    const int wa = f0 + wn * NT * kWideTile, xa = f0 + BN * kWideRow + wm * kWideTile;
    const uint32_t ring_at = __builtin_amdgcn_readfirstlane(uint32_t(reinterpret_cast<uintptr_t>((lds_void*)ring))) + 8 * wave * kWideRow;

    for (int64_t idx = blockIdx.x >> 3; idx < total; idx += gridDim.x >> 3) {
        Item it;
        if (!item_of<MODE, BM>(p, starts, idx, blockIdx.x & 7, &it)) continue;
        // a slice of K is an XCD's, whose L2 then holds that slice of x alone
        const int slice = MODE == kDense ? int(blockIdx.x & 7) % p.ks : 0;
        const int first_step = MODE == kDense ? slice * p.slice_steps : 0;
        const int steps = MODE == kDense ? min(all_steps - first_step, p.slice_steps) : all_steps;
        const int n0 = it.nb * n_step;
        const i32x4 wr = rsrc_words(p.w + it.e * p.w_stride, p.w_extent);
        const uint16_t* xb = p.x;
        uint32_t x_extent = p.x_extent;
        if constexpr (MODE != kUp) {
            xb += (int64_t(it.first) + it.m0) * p.ldx;
            x_extent = uint32_t(tile_bytes(it.mrows, p.ldx, p.K));
        }
        const i32x4 xr = rsrc_words(xb, x_extent);
        uint32_t off[kLoads];      // byte offset of the lane's chunk in slot 0; out of range where there is none
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = 8 * (wave + kWideWaves * i) + (lane >> 3);
            if (i < LW) {     // (a row of the weight for every wave)
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
        // (N: how many of the loads the tile's rows need)
        auto load_slot = [&](auto nc, int step, int slot) {
            constexpr int N = decltype(nc)::value;
            const int kg = step * kWideK;
            // past K out of range, which the top bit says (extents are below 2^31)
            const uint32_t past = kg + 8 * chunk < p.K ? 0u : kOutOfRange;
            const uint32_t to = ring_at + slot * kSlot;
#pragma unroll
            for (int i = 0; i < N; ++i)
                load_to_lds(i < LW ? wr : xr, to + 64 * i * kWideRow, (off[i] + uint32_t(kg) * 2u) | past);
        };
        f32x4 sum[NT][MT];
        Sum64<F64> all[NT][MT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m) sum[t][m] = f32x4{0.f, 0.f, 0.f, 0.f};

        // (the loads counted below are the ring's alone; its slots are free)
        slot_barrier<0>();
        // round r of the walk over K, which may start elsewhere for the next block of columns (rotation); past the last: nothing
        const int start = static_cast<int>(unsigned(it.nb) * unsigned(p.rot) % unsigned(max(steps, 1)));
        auto step_of = [&](int r) { return r >= steps ? all_steps : first_step + (r + start < steps ? r + start : r + start - steps); };
        const int cut = p.K & 7 ? all_steps - 1 : all_steps;     // the step in which K ends within a chunk
        // M of the wave's MT tiles of x
        auto run = [&](auto mc) {
            constexpr int M = decltype(mc)::value;
            constexpr std::integral_constant<int, LW + (16 * WM * M + 63) / 64> n_loads;
            struct Half {
                i32x4 w[NT], x[M];
            };
            auto read = [&](Half& f, int slot, int h) {
                const uint8_t* const at = ring + slot * kSlot;
#pragma unroll
                for (int t = 0; t < NT; ++t) f.w[t] = *reinterpret_cast<const i32x4*>(at + (wa ^ (64 * h)) + t * kWideTile);
#pragma unroll
                for (int m = 0; m < M; ++m) f.x[m] = *reinterpret_cast<const i32x4*>(at + (xa ^ (64 * h)) + m * WM * kWideTile);
            };
            auto multiply = [&](Half& f, int step, int h) {
                if (step == cut) {      // clear what lies past K
                    const int left = p.K - (step * kWideK + 32 * h + 8 * g);
#pragma unroll
                    for (int t = 0; t < NT; ++t) f.w[t] = keep_first(f.w[t], left);
#pragma unroll
                    for (int m = 0; m < M; ++m) f.x[m] = keep_first(f.x[m], left);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int m = 0; m < M; ++m) sum[t][m] = mfma<DT>(f.w[t], f.x[m], sum[t][m]);
            };
#pragma unroll
            for (int s = 0; s < S; ++s) load_slot(n_loads, step_of(s), s);
            slot_barrier<(S - 1) * n_loads.value>();
            Half a, b;
            read(a, 0, 0);
            int slot = 0;
            for (int r = 0; r < steps; ++r) {
                const int step = step_of(r), next = slot == S - 1 ? 0 : slot + 1;
                read(b, slot, 1);
                multiply(a, step, 0);
                // the next slot has landed, and all are done with this one
                slot_barrier<(S - 2) * n_loads.value>();
                load_slot(n_loads, step_of(r + S), slot);
                read(a, next, 0);
                multiply(b, step, 1);
                slot = next;
                if constexpr (F64) {
                    if (r & 1 || r == steps - 1) {
#pragma unroll
                        for (int t = 0; t < NT; ++t)
#pragma unroll
                            for (int m = 0; m < M; ++m) all[t][m].take(sum[t][m]);
                    }
                }
            }
        };
        if (it.mrows <= 16 * WM) run(std::integral_constant<int, 1>{});
        else if (MT == 2 || it.mrows <= 32 * WM) run(std::integral_constant<int, 2>{});
        else if (it.mrows <= 48 * WM) run(std::integral_constant<int, MT - 1>{});
        else run(std::integral_constant<int, MT>{});

        // the sums through the ring's LDS, [m][row of the weight], so that rows of the result are written whole
        slot_barrier<0>();
        float* const tile = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int m = 0; m < MT; ++m)
                *reinterpret_cast<f32x4*>(tile + ((wm + WM * m) * 16 + j) * kPitch + (wn * NT + t) * 16 + 4 * g) = all[t][m].rounded(sum[t][m]);
        slot_barrier<0>();
        constexpr int kWaveRows = BN / WN;
        const int quads = n_step / 4;
        for (int o = tid; o < quads * it.mrows; o += kWideThreads) {
            const int m = o / quads, c = (o - m * quads) * 4, n = n0 + c;
            if (n >= p.N) continue;
            const float* at = tile + m * kPitch;
            at += gated ? c / (kWaveRows / 2) * kWaveRows + c % (kWaveRows / 2) : c;
            const f32x4 v = *reinterpret_cast<const f32x4*>(at);
            f32x4 v2{0.f, 0.f, 0.f, 0.f};
            if (gated) v2 = *reinterpret_cast<const f32x4*>(at + kWaveRows / 2);
            int64_t row = int64_t(it.first) + it.m0 + m;
            if constexpr (MODE == kDown) {
                const int pair = p.pairs[row];
                if (uint32_t(pair) >= uint32_t(p.M)) continue;
                row = pair;
            }
            if (MODE == kDense && p.ks > 1) {              // a slice's sums: finish_kernel adds them
                float* const part = p.part + (int64_t(slice) * p.M + row) * p.ld_part + n;
                *reinterpret_cast<f32x4*>(part) = v;
                if (gated) *reinterpret_cast<f32x4*>(part + p.ld_part / 2) = v2;
                continue;
            }
            float z[4] = {v[0], v[1], v[2], v[3]}, z2[4] = {v2[0], v2[1], v2[2], v2[3]};
            finish4<DT, MODE>(p, row, n, z, z2);
        }
    }
    slot_barrier<0>();       // the ring's last loads into LDS have landed
}

// The slices of K added in order, and what follows: four columns of a row a thread.  (A launch of its own, 5.2 us for four slices of 256 x
// 4096 sums: with the last workgroup of a tile adding them, handed over in the launch, the call took 40 us instead of 33.)
constexpr int kFinishThreads = 256;
template <int DT>
__global__ __launch_bounds__(kFinishThreads) void finish_kernel(const RowsParams p) {
    const int per_row = (p.N + 3) / 4;
    const int64_t i = int64_t(blockIdx.x) * kFinishThreads + threadIdx.x;
    const int64_t row = i / per_row;
    const int n = static_cast<int>(i - row * per_row) * 4;
    if (row >= p.M) return;
    f32x4 a{0.f, 0.f, 0.f, 0.f}, b = a;
    const float* part = p.part + row * p.ld_part + n;
#pragma unroll 4
    for (int q = 0; q < p.ks; ++q, part += int64_t(p.M) * p.ld_part) {
        a += *reinterpret_cast<const f32x4*>(part);
        if (p.gated) b += *reinterpret_cast<const f32x4*>(part + p.ld_part / 2);
    }
    float z[4] = {a[0], a[1], a[2], a[3]}, z2[4] = {b[0], b[1], b[2], b[3]};
    finish4<DT, kDense>(p, row, n, z, z2);
}

}  // namespace rows
}  // namespace nmm
