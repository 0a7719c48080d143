// Products with weights given as [N, K] whose rows of x and whose results are addressed one by one, and what follows them
// in the same launch (device code):
//   kDense   y[m] = act(x[m] Wt^T + bias) + residual, or the gated form             (nt_act.hip)
//   kUp      h[s] = act(x[t] Wg^T) * (x[t] Wu^T), pair s of the order by experts     (moe_experts.hip)
//   kDown    part[p] = h[s] W2^T, p = pairs[s]                                       (moe_experts.hip)
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "bf16_cast.h"
#include "moe_tiles.h"
#include "nmm_internal.h"
#include "nt_ring.h"

namespace nmm {
namespace rows {

using namespace ring;

enum Mode { kDense, kUp, kDown };

constexpr int kMaxExperts = 1024;
constexpr int kRedPitch = 20;                   // floats of one m in a 16 x 16 tile of sums in LDS
constexpr int kTileFloats = 16 * kRedPitch;

struct RowsParams {
    const uint16_t* x;
    int64_t ldx;                 // elements
    const uint8_t* w;
    int64_t w_stride;            // bytes from one expert's matrix to the next
    uint32_t row_bytes, w_extent;
    uint32_t x_extent;           // kUp: bytes of x
    int K, N;
    int M;                       // rows of x (kDense), pairs (kUp, kDown)
    int n_blocks;
    int gated, act;
    const uint16_t* bias;        // or NULL
    const uint16_t* res;         // or NULL
    int64_t ldr;
    uint16_t* y;                 // kDense: or NULL; kUp: h
    int64_t ldy;
    float* yf;                   // kDense: or NULL; kDown: part
    int64_t ldyf;
    const int32_t* offsets;      // those of the first expert here
    const int32_t* pairs;
    int local, top_k;
    int ks, slice_steps;         // wide tiles of kDense: K in ks slices of slice_steps slots
    float* part;                 // their sums: [ks][M][ld_part], a gate's columns, then those that it multiplies
    int64_t ld_part;
    int rot;                     // rounds by which the next block of columns starts its walk over K later
};

// Rows of the weight a multiple of 4 KB apart meet in few of the memory's channels, as all workgroups are at about the same k:
// there the next block of columns starts its walk over K a round later (16 experts of 2048 x 7168, 16 rows each: 114 -> 94 us; 32 x
// 16384 x 7168: 48 -> 45; 128 rows each 138 -> 131.5, though each L2 then reads h about four times, 0.73 instead of 0.55 GB in all: an expert's
// workgroups are at different k, and W passes through L2 between them).  Elsewhere it only takes from L2 what workgroups at the same k share (7168 x 2 x 2048: 250 -> 259 us).
inline int rotation(int64_t ld) { return ld * 2 % 4096 == 0 ? 1 : 0; }

__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case NMM_ACT_RELU: return z < 0.f ? 0.f : z;
        case NMM_ACT_SILU: return z / (1.f + expf(-z));
        case NMM_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678118654752f);
        // (1 + tanh u) / 2 = 1 / (1 + e^-2u)
        case NMM_ACT_GELU_TANH: return z / (1.f + expf(-1.5957691216057308f * (z + 0.044715f * z * z * z)));
        default: return z;
    }
}

template <int DT>
__device__ __forceinline__ float up16(uint16_t b) {
    if constexpr (DT == NMM_BF16) return __uint_as_float(uint32_t(b) << 16);
    else return float(__builtin_bit_cast(_Float16, b));
}
template <int DT>
__device__ __forceinline__ uint16_t down16(float v) {
    if constexpr (DT == NMM_BF16) return to_bf16_bits(v);
    else return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
}

// v to row[n .. n + 3], columns at or past N left alone.
template <int DT>
__device__ __forceinline__ void store4(uint16_t* row, int n, int N, const float (&v)[4]) {
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = down16<DT>(v[i]);
    if (n + 4 <= N && (reinterpret_cast<uintptr_t>(row + n) & 7u) == 0) {
        *reinterpret_cast<uint2*>(row + n) =
            uint2{uint32_t(h[0]) | (uint32_t(h[1]) << 16), uint32_t(h[2]) | (uint32_t(h[3]) << 16)};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) row[n + i] = h[i];
}
__device__ __forceinline__ void store4(float* row, int n, int N, const float (&v)[4]) {
    if (n + 4 <= N && (reinterpret_cast<uintptr_t>(row + n) & 15u) == 0) {
        *reinterpret_cast<f32x4*>(row + n) = f32x4{v[0], v[1], v[2], v[3]};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (n + i < N) row[n + i] = v[i];
}

// What follows the product for four columns n .. n + 3 of row m of the tile (z, and z2 of the up rows).
template <int DT, int MODE>
__device__ __forceinline__ void finish4(const RowsParams& p, int64_t row, int n, float (&z)[4], float (&z2)[4]) {
    if constexpr (MODE == kDown) {
        store4(p.yf + row * p.ldyf, n, p.N, z);
        return;
    }
    if constexpr (MODE == kDense) {
        if (p.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) {
                    z[i] += up16<DT>(p.bias[n + i]);
                    if (p.gated) z2[i] += up16<DT>(p.bias[p.N + n + i]);
                }
        }
    }
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = activate(z[i], p.act);
        if (MODE == kUp || p.gated) v[i] *= z2[i];
    }
    if constexpr (MODE == kDense) {
        if (p.res) {
            const uint16_t* r = p.res + row * p.ldr;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < p.N) v[i] += up16<DT>(r[n + i]);
        }
        if (p.yf) store4(p.yf + row * p.ldyf, n, p.N, v);
        if (!p.y) return;
    }
    store4<DT>(p.y + row * p.ldy, n, p.N, v);
}

// The tiles of TM rows of each expert here: starts[e] counts those of the experts before e.
template <int TM, int THREADS>
__device__ __forceinline__ void scan_tiles(const RowsParams& p, int* starts) {
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        const int most = most_tiles(p.M, TM, p.local);
        int carry = 0;
        if (lane == 0) starts[0] = 0;
        for (int e0 = 0; e0 < p.local; e0 += 64) {
            const int e = e0 + lane;
            int c = 0;
            if (e < p.local) c = tiles_of(cut_offset(p.offsets[e], p.M), cut_offset(p.offsets[e + 1], p.M), TM);
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(c, d);
                if (lane >= d) c += o;
            }
            if (e < p.local) starts[e + 1] = min(carry + c, most);      // (64 experts have less than 2^31 tiles)
            carry = min(carry + __shfl(c, 63), most);
        }
    }
    __syncthreads();
}

// One item: an expert, a tile of its rows and a block of output columns.
struct Item {
    int e, first, m0, mrows, nb;      // first: the expert's first pair in the order by experts
};

__device__ __forceinline__ int64_t blocks_of(const RowsParams& p) { return blocks_of_xcd(p.n_blocks, p.ks); }

// Item idx of this XCD (false: none): its blocks of columns of all experts, so that each XCD has the same share of every
// expert's rows.  (An eighth of the experts each reads x into one L2 instead of eight, 0.95 instead of 1.12 GB for 16 experts of 128 rows on
// average, but the XCD with the fullest ones ends last: 253 instead of 228 us.)
template <int MODE, int TM>
__device__ __forceinline__ bool item_of(const RowsParams& p, const int* starts, int64_t idx, int xcd, Item* it) {
    int tiles, count;
    int64_t rem = idx;
    it->e = 0;
    it->first = 0;
    if constexpr (MODE == kDense) {
        tiles = static_cast<int>((int64_t(p.M) + TM - 1) / TM);
        count = p.M;
    } else {
        const int64_t nb8 = blocks_of(p);
        const int e = __builtin_amdgcn_readfirstlane(expert_of(starts, p.local, static_cast<int>(idx / nb8)));
        const int s = __builtin_amdgcn_readfirstlane(starts[e]);
        tiles = __builtin_amdgcn_readfirstlane(starts[e + 1]) - s;
        rem = idx - s * nb8;
        it->e = e;
        it->first = __builtin_amdgcn_readfirstlane(cut_offset(p.offsets[e], p.M));
        count = __builtin_amdgcn_readfirstlane(cut_offset(p.offsets[e + 1], p.M)) - it->first;
    }
    const Place at = place_of(rem, tiles, TM, p.ks, xcd);
    it->nb = at.nb;
    it->m0 = at.m0;
    it->mrows = min(TM, count - it->m0);
    return it->nb < p.n_blocks;
}

// A lane's four values of a tile summed in fp64, where F64: what the matrix cores have added up in fp32 so far is taken into it.
template <bool F64>
struct Sum64 {
    __device__ __forceinline__ f32x4 rounded(f32x4 sum) const { return sum; }
};
template <>
struct Sum64<true> {
    double v[4] = {0.0, 0.0, 0.0, 0.0};
    __device__ __forceinline__ void take(f32x4& sum) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += double(sum[i]);
        sum = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ f32x4 rounded(f32x4) const { return f32x4{float(v[0]), float(v[1]), float(v[2]), float(v[3])}; }
};

// Few rows of x a tile (4 XR): a workgroup owns 16 NT rows of the weight (gated: half of them the gate's, half those that they are
// multiplied with) and all of K, which its NW waves share in groups of 128, as in mfma_nt_kernel: rings of D groups private to a
// wave, no barrier in the loop.  Sums are fp32 in the matrix cores, two chains a wave, the waves' added in wave order: relative 2-norm
// error 2.7e-7 (16 rows of the weight, four waves) and 4.0e-7 (32, two) at K = 16384.  A y of 16 bits hides that; where results are asked for in
// fp32 (F64), a wave takes its sums of two matrix instructions each into fp64, as mfma_nt_kernel does: 5.6e-8 (fp16 7.0e-8), 32 rows x 16384 x
// 7168 45.1 us instead of 43.5, the others as fast.
// What bounds it: the weight's bytes, read once.  32 rows x 16384 x 7168 45 us (5.2 TB/s), eight experts' W1 of 2 x 2048 x 7168 for one
// token 67 (7.0 TB/s), 64 experts' for 64 tokens 581 (6.5 TB/s), where a copy moves 5.0; a weight of 59 MB 12 us, of which 2 are a launch
// and 2 the first loads.
template <int DT, int MODE, int XR, int NT, int NW, bool F64 = false>
__global__ __launch_bounds__(64 * NW) void rows_kernel(const RowsParams p) {
    constexpr int D = 2;                             // groups of a ring
    constexpr int TM = 4 * XR;
    constexpr int MT = XR > 4 ? 2 : 1;               // 16-row tiles of x
    constexpr int kLoads = 4 * NT + XR;              // loads of a group per wave
    constexpr int kSlot = kLoads * kQuad;            // LDS bytes of a group
    __shared__ __attribute__((aligned(256))) uint8_t smem[NW * D * kSlot];
    __shared__ __attribute__((aligned(16))) float red[NW * NT * MT * kTileFloats];
    __shared__ int starts[MODE == kDense ? 1 : kMaxExperts + 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, j = lane & 15;
    const bool gated = MODE == kUp || (MODE == kDense && p.gated);
    const int n_step = gated ? 8 * NT : 16 * NT;

    if constexpr (MODE != kDense) scan_tiles<TM, 64 * NW>(p, starts);
    const int64_t nb8 = blocks_of(p);
    const int64_t total = (MODE == kDense ? (int64_t(p.M) + TM - 1) / TM : int64_t(__builtin_amdgcn_readfirstlane(starts[p.local]))) * nb8;
    const int groups = (p.K + kMfmaNtGroup - 1) / kMfmaNtGroup;
    const int rounds = (groups + NW - 1) / NW;       // the same for every wave; groups past K are zeros
    uint8_t* const ring = smem + wave * (D * kSlot);
    // LDS addresses of the lane's fragment of step 0: row j, chunk g; step s flips bits 6 and 7
    const uint32_t base = uint32_t(reinterpret_cast<uintptr_t>((lds_void*)ring));
    const uint32_t wa = base + uint32_t(j * kRowBytes + ((g ^ j) * 16));
    const int jx = XR < 4 ? (j & (4 * XR - 1)) : j;
    const uint32_t xa = base + uint32_t(jx * kRowBytes + ((g ^ jx) * 16));

    for (int64_t idx = blockIdx.x >> 3; idx < total; idx += gridDim.x >> 3) {
        Item it;
        if (!item_of<MODE, TM>(p, starts, idx, blockIdx.x & 7, &it)) continue;
        const int n0 = it.nb * n_step;
        const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<uint8_t*>(p.w + it.e * p.w_stride), (short)0, (int)p.w_extent, kRsrcWord3);
        const uint16_t* xb = p.x;
        uint32_t x_extent = p.x_extent;
        if constexpr (MODE != kUp) {
            xb += (int64_t(it.first) + it.m0) * p.ldx;
            x_extent = uint32_t(tile_bytes(it.mrows, p.ldx, p.K));
        }
        const __amdgpu_buffer_rsrc_t xr =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(xb), (short)0, (int)x_extent, kRsrcWord3);
        // Load q of a group covers rows 4 q .. 4 q + 3, lane l the slot l % 16 of row 4 q + l / 16.  Slot c of row r
        // holds the row's chunk c ^ (r % 16), so that the 16 rows of a fragment read lie in 16 different 16-byte columns.
        uint32_t off[kLoads];      // byte offset of the lane's chunk in group 0; out of range where there is none
        int kc[4];                 // its first k in group 0, by row quad of a tile
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const bool is_w = q < 4 * NT;
            const int r = 4 * (is_w ? q : q - 4 * NT) + g;
            const int c = j ^ (r & 15);
            if (q < 4) kc[q] = 8 * c;
            if (is_w) {
                constexpr int kHalf = 8 * NT;         // gated: the gate's rows, then as many that they are multiplied with
                const int n = gated ? n0 + r % kHalf : n0 + r;
                const int64_t row = gated && r >= kHalf ? int64_t(p.N) + n : n;
                off[q] = n < p.N ? uint32_t(row * p.row_bytes) + 16u * c : kOutOfRange;
            } else {
                bool ok = r < it.mrows;
                int64_t row = r;
                if constexpr (MODE == kUp) {
                    const int pair = ok ? p.pairs[it.first + it.m0 + r] : -1;
                    ok = uint32_t(pair) < uint32_t(p.M);
                    row = pair / p.top_k;
                }
                off[q] = ok ? uint32_t(row * p.ldx * 2) + 16u * c : kOutOfRange;
            }
        }
        auto load_group = [&](int group, uint8_t* slot) {
            const int kg = group * kMfmaNtGroup;
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const int qq = q < 4 * NT ? q & 3 : (q - 4 * NT) & 3;
                const uint32_t o = (kg + kc[qq] < p.K) ? off[q] + uint32_t(kg) * 2u : kOutOfRange;
                if (q < 4 * NT)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(wr, (lds_void*)(slot + q * kQuad), 16, o, 0, 0, kLoadNT);
                else
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(xr, (lds_void*)(slot + q * kQuad), 16, o, 0, 0, 0);
            }
        };
        const int start = static_cast<int>(unsigned(it.nb) * unsigned(p.rot) % unsigned(max(rounds, 1)));
        auto group_of = [&](int r) { return r < rounds ? wave + (r + start < rounds ? r + start : r + start - rounds) * NW : groups; };
        // (the loads counted below are the ring's alone)
        __builtin_amdgcn_s_waitcnt(0);
#pragma unroll
        for (int d = 0; d < D; ++d) load_group(group_of(d), ring + d * kSlot);

        f32x4 sum[NT][MT][2];
        Sum64<F64> all[NT][MT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sum[t][mt][0] = sum[t][mt][1] = f32x4{0.f, 0.f, 0.f, 0.f};

        auto consume = [&](auto dc, int r) {
            constexpr int d = decltype(dc)::value;
            constexpr int kOff = d * kSlot, kXOff = kOff + 4 * NT * kQuad;
            const int group = group_of(r);
            const bool ragged = (group + 1) * kMfmaNtGroup > p.K;
            auto half = [&](auto hc) {
                constexpr int h = decltype(hc)::value;
                i32x4 w0[NT], w1[NT], x0[MT], x1[MT];
                read_pair<(D - 1) * kLoads, NT, MT, kOff, kXOff>(w0, w1, x0, x1, wa ^ (128u * h), wa ^ (128u * h + 64u),
                                                                 xa ^ (128u * h), xa ^ (128u * h + 64u));
                if (ragged) {   // clear what lies past K
                    const int l0 = p.K - (group * kMfmaNtGroup + 64 * h + 8 * g), l1 = l0 - 32;
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        w0[t] = keep_first(w0[t], l0);
                        w1[t] = keep_first(w1[t], l1);
                    }
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        x0[mt] = keep_first(x0[mt], l0);
                        x1[mt] = keep_first(x1[mt], l1);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        sum[t][mt][0] = mfma<DT>(w0[t], x0[mt], sum[t][mt][0]);
                        sum[t][mt][1] = mfma<DT>(w1[t], x1[mt], sum[t][mt][1]);
                    }
            };
            half(std::integral_constant<int, 0>{});
            half(std::integral_constant<int, 1>{});
            load_group(group_of(r + D), ring + kOff);
            if constexpr (F64) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        all[t][mt].take(sum[t][mt][0]);
                        all[t][mt].take(sum[t][mt][1]);
                    }
            }
        };
        for (int r = 0; r < rounds; r += D) {
            consume(std::integral_constant<int, 0>{}, r);
            if (r + 1 < rounds) consume(std::integral_constant<int, 1>{}, r + 1);
        }

        // the waves' sums through LDS: lane (g, j) holds n = 4 g + i, m = j of each tile
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                *reinterpret_cast<f32x4*>(red + ((wave * NT + t) * MT + mt) * kTileFloats + j * kRedPitch + 4 * g) =
                    all[t][mt].rounded(sum[t][mt][0] + sum[t][mt][1]);
        __syncthreads();
        const int quads = n_step / 4;
        for (int o = tid; o < quads * it.mrows; o += 64 * NW) {
            const int q = o % quads, m = o / quads;
            const float* src = red + ((q >> 2) * MT + (m >> 4)) * kTileFloats + (m & 15) * kRedPitch + 4 * (q & 3);
            float z[4], z2[4] = {0.f, 0.f, 0.f, 0.f};
            f32x4 a{0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                a += *reinterpret_cast<const f32x4*>(src + w * NT * MT * kTileFloats);
                if (gated) b += *reinterpret_cast<const f32x4*>(src + (NT > 1 ? (w * NT + 1) * MT * kTileFloats : w * MT * kTileFloats + 8));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[i] = a[i];
                z2[i] = b[i];
            }
            const int n = n0 + 4 * q;
            int64_t row = int64_t(it.first) + it.m0 + m;
            if constexpr (MODE == kDown) {
                const int pair = p.pairs[row];
                if (uint32_t(pair) >= uint32_t(p.M)) continue;
                row = pair;
            }
            if (n < p.N) finish4<DT, MODE>(p, row, n, z, z2);
        }
        __syncthreads();           // red and the rings are the next item's
    }
}

}  // namespace rows
}  // namespace nmm
