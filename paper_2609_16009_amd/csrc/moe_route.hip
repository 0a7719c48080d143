// Routing to experts: scores, the choice of each token, and the (token, expert) pairs in the order of the experts.
//
// LPT lanes take a token, lane l of them the experts l PER .. l PER + PER - 1, all in fp64: which expert comes before which may
// not depend on how a score was rounded.  Choosing is top_k rounds of a maximum over 64-bit keys that order as the values do
// (upper halves, then lower ones among their equals, then the lowest index), 0 for what has been chosen or lies in a closed
// group.  A wave a token (LPT 64) has the shorter chain, four tokens a wave share every step's instructions.
//
// The pairs are sorted by counting: a wave walks its stretch of pairs, 64 at a time, and learns from one ballot per bit of the
// expert's number which lanes hold the same one, so that a pair's place is its expert's next place plus its rank among them.
// Up to kOneLaunch pairs the last workgroup to finish its tokens does it (handoff.h), with more a second launch, to which
// each workgroup of the first leaves the counts of its tokens.
//
// What bounds it: for few tokens the chain of dependent steps, top_k maxima over a wave among them (one token, 8 of 256 experts
// in groups, 6.5 us; 64 tokens 11.1 with the hand-over); for many the maxima's instructions (32767 tokens, 6 of 60 experts: 13 us of 22.5)
// and the places (8.6, of which 4.1 are that each workgroup first adds up what all of them counted, 512 times 512 rows out of L2).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "handoff.h"
#include "nmm_internal.h"
#include "wave64.h"

namespace nmm {
namespace {

constexpr int kRouteWaves = 8, kRouteThreads = 64 * kRouteWaves;
// Pairs ordered in the first launch (1020 pairs of 60 experts 7.7 us, 9.8 in two launches; 1024 of 256 12.0 and 12.9), while they fit LDS.
constexpr int64_t kOneLaunch = 1024;
constexpr int64_t kSharedWaves = 2048;  // tokens from which four share a wave
constexpr int64_t kPiece = 4096;      // pairs of a segment ordered at a time
// Workgroups of the first launch: each of the second reads the counts of all of them (32767 tokens of 60 experts 22.3 us with 512, 23.5 with
// 256, 35 with 128; 8192 of 256 experts 34.5, 32.9, 53).
constexpr int64_t max_segments(int64_t experts) { return experts <= 64 ? 512 : 256; }
constexpr int kMaxRouted = 1024;      // experts
constexpr int kFewPairs = kRouteWaves * 32;
constexpr uint16_t kNoExpert = 0xFFFF;

struct RouteParams {
    const void* logits;
    int64_t ld;
    const float* bias;
    const uint8_t* mask;
    int32_t* chosen;
    float* weights;
    int32_t* offsets;
    int32_t* pairs;
    unsigned* arrived;
    int32_t* counts;          // [segments][experts_up], more than kOneLaunch pairs
    double scale;
    int tokens, experts, top_k;
    int groups, group_size, top_groups, group_top, group_lanes;
    int bf16, sigmoid, renormalize, wide;
    int segments;             // 0: the pairs are ordered in the first launch
    int chunk;                // tokens of a workgroup
    int experts_up;           // experts rounded up to a multiple of 4
};

// LDS of a wave written by some of its lanes and read by others.
__device__ __forceinline__ void wave_lds_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
    return __builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, false);
}

// The maximum over LPT lanes in each of them.
template <int LPT>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    x = max(x, dpp_u32<0xB1>(x));
    x = max(x, dpp_u32<0x4E>(x));
    x = max(x, dpp_u32<0x141>(x));
    x = max(x, dpp_u32<0x140>(x));
    if constexpr (LPT == 64) {
        const wave_u32x2 a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = max(a[0], a[1]);
        const wave_u32x2 b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = max(b[0], b[1]);
    }
    return x;
}
template <int LPT>
__device__ __forceinline__ double lanes_max(double x) {
    if constexpr (LPT == 64) return max64(x);
    x = __builtin_fmax(x, dpp_move<0xB1>(x));
    x = __builtin_fmax(x, dpp_move<0x4E>(x));
    x = __builtin_fmax(x, dpp_move<0x141>(x));
    return __builtin_fmax(x, dpp_move<0x140>(x));
}
template <int LPT>
__device__ __forceinline__ double lanes_sum(double x) {
    if constexpr (LPT == 64) return sum64(x);
    x += dpp_move<0xB1>(x);
    x += dpp_move<0x4E>(x);
    x += dpp_move<0x141>(x);
    return x + dpp_move<0x140>(x);
}

// The best two of two lanes' best two.
__device__ __forceinline__ void best_two(double& best, double& second, double ob, double os) {
    second = __builtin_fmax(__builtin_fmin(best, ob), __builtin_fmax(second, os));
    best = __builtin_fmax(best, ob);
}
template <int CTRL>
__device__ __forceinline__ void best_two_dpp(double& best, double& second) {
    best_two(best, second, dpp_move<CTRL>(best), dpp_move<CTRL>(second));
}

// e^x to about 2^-52 of it: x = k ln 2 + r with ln 2 in two parts, Taylor's series of e^r to r^13 (|r| <= ln 2 / 2: the rest is
// below 2^-58), times 2^k.
__device__ __forceinline__ double exp64(double x) {
    x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;       // (NaN stays)
    const double k = __builtin_rint(x * 1.4426950408889634);
    const double r = fma(-k, 2.3190468138462996e-17, fma(-k, 0.6931471805599453, x));
    double y = 1.0 / 6227020800.0;
    y = fma(y, r, 1.0 / 479001600.0);
    y = fma(y, r, 1.0 / 39916800.0);
    y = fma(y, r, 1.0 / 3628800.0);
    y = fma(y, r, 1.0 / 362880.0);
    y = fma(y, r, 1.0 / 40320.0);
    y = fma(y, r, 1.0 / 5040.0);
    y = fma(y, r, 1.0 / 720.0);
    y = fma(y, r, 1.0 / 120.0);
    y = fma(y, r, 1.0 / 24.0);
    y = fma(y, r, 1.0 / 6.0);
    y = fma(y, r, 0.5);
    y = fma(y, r, 1.0);
    y = fma(y, r, 1.0);
    return __builtin_ldexp(y, int(k));
}

// 1 / d for d >= 1 (infinity: 0; NaN stays): the instruction's estimate and two Newton steps.
__device__ __forceinline__ double inverse(double d) {
    double y = __builtin_amdgcn_rcp(d);
    y = fma(fma(-d, y, 1.0), y, y);
    y = fma(fma(-d, y, 1.0), y, y);
    return d == INFINITY ? 0.0 : y;
}

// The value of another lane.
__device__ __forceinline__ double lane_of(double x, int lane) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_ds_bpermute(lane << 2, int(uint32_t(u)));
    const uint32_t hi = __builtin_amdgcn_ds_bpermute(lane << 2, int(uint32_t(u >> 32)));
    return __longlong_as_double((uint64_t(hi) << 32) | lo);
}

// The bits of c, ordered as unsigned numbers the way the values are (0: below all of them; c is not NaN).
__device__ __forceinline__ uint64_t order_key(double c) {
    const uint64_t u = __double_as_longlong(c + 0.0);        // (-0 and 0 are equal)
    return u ^ (uint64_t(int64_t(u) >> 63) | 0x8000000000000000ull);
}

// Whether each 16 of the bits hold a single one.
__device__ __forceinline__ bool one_each(uint64_t bits) {
    uint64_t more = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = uint32_t(bits >> (16 * i)) & 0xFFFFu;
        more |= b & (b - 1);
    }
    return more == 0;
}

// Scores s and, by what they are chosen, c of the lane's experts of token t; NaN where there is no expert.
template <int LPT, int PER>
__device__ __forceinline__ void scores(const RouteParams& p, int64_t t, int l, double (&s)[PER], double (&c)[PER]) {
    const double nan = __longlong_as_double(0x7FF8000000000000ll);
    const int e0 = l * PER;
    float v[PER];
    bool done = false;
    if constexpr (PER % 4 == 0) {
        if (p.wide) {
            done = true;
#pragma unroll
            for (int q = 0; q < PER / 4; ++q) {
                if (e0 + 4 * q >= p.experts) continue;
                if (p.bf16) {
                    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.logits) + t * p.ld + e0 + 4 * q);
                    v[4 * q] = __uint_as_float(u.x << 16);
                    v[4 * q + 1] = __uint_as_float(u.x & 0xFFFF0000u);
                    v[4 * q + 2] = __uint_as_float(u.y << 16);
                    v[4 * q + 3] = __uint_as_float(u.y & 0xFFFF0000u);
                } else {
                    const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(p.logits) + t * p.ld + e0 + 4 * q);
                    v[4 * q] = f.x;
                    v[4 * q + 1] = f.y;
                    v[4 * q + 2] = f.z;
                    v[4 * q + 3] = f.w;
                }
            }
        }
    }
    if (!done) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (e0 + i < p.experts)
                v[i] = p.bf16 ? __uint_as_float(uint32_t(static_cast<const uint16_t*>(p.logits)[t * p.ld + e0 + i]) << 16)
                              : static_cast<const float*>(p.logits)[t * p.ld + e0 + i];
    }
    float b[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) b[i] = p.bias && e0 + i < p.experts ? p.bias[e0 + i] : 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) s[i] = e0 + i < p.experts ? double(v[i]) : nan;
    if (p.sigmoid) {
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] = inverse(1.0 + exp64(-s[i]));
    } else {
        double top = s[0], sum = 0.0;
#pragma unroll
        for (int i = 1; i < PER; ++i) top = __builtin_fmax(top, s[i]);
        top = lanes_max<LPT>(top);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            s[i] = exp64(s[i] - top);
            if (e0 + i < p.experts) sum += s[i];
        }
        sum = 1.0 / lanes_sum<LPT>(sum);
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i] *= sum;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        c[i] = p.bias ? s[i] + double(b[i]) : s[i];
        if (c[i] != c[i]) c[i] = -INFINITY;
    }
}

// Counts of the experts in choices from .. to of this wave.
__device__ __forceinline__ void count_choices(const uint16_t* choices, int from, int to, int* counts) {
    for (int i = from + (threadIdx.x & 63); i < to; i += 64) {
        const uint32_t e = choices[i];
        if (e != kNoExpert) atomicAdd(counts + e, 1);
    }
}

// Choices from .. to of this wave to their places; next[e]: the next place of expert e; `first`: the number of pair 0.
__device__ __forceinline__ void place_choices(const RouteParams& p, const uint16_t* choices, int from, int to, int first, int* next) {
    const int lane = threadIdx.x & 63;
    const int bits = 32 - __builtin_clz(p.experts);
    for (int i0 = from; i0 < to; i0 += 64) {
        const int i = i0 + lane;
        const uint32_t e = i < to ? choices[i] : kNoExpert;
        uint64_t same = __builtin_amdgcn_ballot_w64(e != kNoExpert);
        for (int b = 0; b < bits; ++b) {
            const uint64_t ones = __builtin_amdgcn_ballot_w64((e >> b) & 1);
            same &= (e >> b) & 1 ? ones : ~ones;
        }
        const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
        const int at = e != kNoExpert ? next[e] : 0;
        wave_lds_sync();
        if (e != kNoExpert) {
            p.pairs[at + rank] = first + i;
            if (rank == 0) next[e] = at + __builtin_popcountll(same);
        }
        wave_lds_sync();
    }
}

// base[e], pairs of expert e that lie ahead of these ones, becomes their first place: all[] holds how many pairs each expert
// has in total, and experts follow each other.  By the first wave, lane l the experts l per .. l per + per - 1.  Where
// `offsets` is given, it is written.
__device__ __forceinline__ void scan_experts(const RouteParams& p, const int* all, int* base, int32_t* offsets) {
    const int lane = threadIdx.x & 63, per = (p.experts + 63) / 64;
    const int e0 = min(lane * per, p.experts), e1 = min(e0 + per, p.experts);
    int sum = 0;
    for (int e = e0; e < e1; ++e) sum += all[e];
    int start = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(start, d);
        if (lane >= d) start += o;
    }
    if (offsets && lane == 63) offsets[p.experts] = start;
    start -= sum;
    for (int e = e0; e < e1; ++e) {
        if (offsets) offsets[e] = start;
        base[e] += start;
        start += all[e];
    }
}

// Counts of n choices in each wave's stretch (whole 64s) of them.
__device__ __forceinline__ void count_piece(const RouteParams& p, const uint16_t* choices, int n, int* counts, int* from, int* to) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < kRouteWaves * p.experts; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    const int each = (n + kRouteThreads - 1) / kRouteThreads * 64;
    *from = min(wave * each, n);
    *to = min(*from + each, n);
    count_choices(choices, *from, *to, counts + wave * p.experts);
    __syncthreads();
}

// They become places from base[] on, which moves behind the last.
__device__ __forceinline__ void places_of_piece(const RouteParams& p, int* counts, int* base) {
    for (int e = threadIdx.x; e < p.experts; e += kRouteThreads) {
        int n[kRouteWaves], at = base[e];
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) n[w] = counts[w * p.experts + e];
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) {
            counts[w * p.experts + e] = at;
            at += n[w];
        }
        base[e] = at;
    }
    __syncthreads();
}

// n pairs, kFewPairs at most, counted pair by pair: a pair's place is the number of pairs ahead of it, an expert's first place
// that of the pairs with lower experts.  choices: read whole, a thread's own included.
__device__ __forceinline__ void order_few(const RouteParams& p, const uint16_t* choices, int n) {
    for (int i = threadIdx.x; i < n + p.experts + 1; i += kRouteThreads) {
        const bool pair = i < n;
        const uint32_t e = pair ? choices[i] : uint32_t(i - n);
        const int later = pair ? i : 0;
        int ahead = 0;
#pragma unroll 8
        for (int k = 0; k < n; ++k) {
            const uint32_t o = choices[k];
            ahead += o < e || (o == e && k < later) ? 1 : 0;
        }
        if (!pair) p.offsets[e] = ahead;
        else if (e != kNoExpert) p.pairs[ahead] = i;
    }
}

// All n pairs by one workgroup.  lds: [waves + 2][experts].
__device__ __forceinline__ void order_all(const RouteParams& p, const uint16_t* choices, int n, int* lds) {
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int* const all = lds + kRouteWaves * p.experts;
    int* const base = all + p.experts;
    int from, to;
    count_piece(p, choices, n, lds, &from, &to);
    for (int e = tid; e < p.experts; e += kRouteThreads) {
        int v = 0;
#pragma unroll
        for (int w = 0; w < kRouteWaves; ++w) v += lds[w * p.experts + e];
        all[e] = v;
        base[e] = 0;
    }
    __syncthreads();
    if (wave == 0) scan_experts(p, all, base, p.offsets);
    __syncthreads();
    places_of_piece(p, lds, base);
    place_choices(p, choices, from, to, 0, lds + wave * p.experts);
}

// LDS: a wave's scores of its tokens; then, in the last workgroup, the choices and their counts.
template <int LPT, int PER>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t route_lds[];
    __shared__ uint16_t few[kFewPairs];         // the choices of a single workgroup's tokens
    __shared__ int last;
    constexpr int TPW = 64 / LPT;
    const int tid = threadIdx.x, lane = tid & 63, l = lane % LPT;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    double* const mine = reinterpret_cast<double*>(route_lds) + (wave * TPW + lane / LPT) * p.experts;
    int* const seg_counts = reinterpret_cast<int*>(route_lds + size_t(kRouteWaves) * TPW * p.experts * 8);
    const bool one = gridDim.x == 1;
    if (p.segments) {
        for (int e = tid; e < p.experts_up; e += kRouteThreads) seg_counts[e] = 0;
        __syncthreads();
    }
    const int t0 = static_cast<int>(blockIdx.x) * p.chunk, t1 = min(t0 + p.chunk, p.tokens);
    for (int tb = t0 + wave * TPW; tb < t1; tb += kRouteWaves * TPW) {
        const int t = tb + lane / LPT;
        const bool there = t < t1;
        const bool live = there && !(p.mask && p.mask[t] == 0);
        double s[PER], c[PER];
        scores<LPT, PER>(p, there ? t : tb, l, s, c);
        uint64_t open = ~uint64_t(0);             // of the token's groups
        if (p.groups > 1) {
            // group_lanes lanes share a group: its best two, then its rank among the groups
            const int gl = p.group_lanes, grp = l / gl, sub = l % gl;
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (l * PER + i < p.experts) mine[l * PER + i] = c[i];
            wave_lds_sync();
            double best = -INFINITY, second = -INFINITY;
            if (grp < p.groups) {
#pragma unroll 4
                for (int i = sub; i < p.group_size; i += gl) best_two(best, second, mine[grp * p.group_size + i], -INFINITY);
            }
            if (gl > 1) best_two_dpp<0xB1>(best, second);
            if (gl > 2) best_two_dpp<0x4E>(best, second);
            if (gl > 4) best_two_dpp<0x141>(best, second);
            if (gl > 8) best_two_dpp<0x140>(best, second);
            if (gl > 16) {
                double a, b, d, e;
                row_pair16(best, &a, &b);
                row_pair16(second, &d, &e);
                best = a;
                second = d;
                best_two(best, second, b, e);
            }
            double total = p.group_top == 2 && p.group_size > 1 ? best + second : best;
            if (total != total) total = -INFINITY;
            wave_lds_sync();
            if (grp < p.groups && sub == 0) mine[grp] = total;
            wave_lds_sync();
            int ahead = 0;
#pragma unroll 4
            for (int o = 0; o < p.groups; ++o) {
                const double v = mine[o];
                ahead += v > total || (v == total && o < grp) ? 1 : 0;
            }
            const uint64_t ranked = __builtin_amdgcn_ballot_w64(grp < p.groups && ahead < p.top_groups) >> (lane - l);
            // (bit grp * group_lanes and the lanes behind it stand for group grp)
            open = ranked;
            wave_lds_sync();
        }
        uint64_t key[PER];
        {
            int grp = 0, left = p.experts;
            if (p.groups > 1) {
                grp = l * PER / p.group_size;
                left = (grp + 1) * p.group_size - l * PER;
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = l * PER + i;
                if (left == 0) {
                    ++grp;
                    left = p.group_size;
                }
                --left;
                const bool in = e < p.experts && ((open >> ((grp * p.group_lanes) & 63)) & 1);
                const uint64_t k = order_key(c[i]);
                key[i] = in ? k : 0;
                if (e < p.experts) mine[e] = s[i];
            }
        }
        uint32_t my_e = 0;
        for (int i = 0; i < p.top_k; ++i) {
            uint64_t best = key[0];
            uint32_t at = 0;
#pragma unroll
            for (int k = 1; k < PER; ++k) {
                const bool more = key[k] > best;
                best = more ? key[k] : best;
                at = more ? k : at;
            }
            const uint32_t bh = uint32_t(best >> 32), bl = uint32_t(best);
            const uint32_t mh = lanes_max<LPT>(bh);
            // nearly always one lane of a token holds the largest upper half
            bool holds = bh == mh;
            uint64_t holders = __builtin_amdgcn_ballot_w64(holds);
            uint32_t e;
            if (LPT == 64 && (holders & (holders - 1)) == 0) {
                e = __builtin_amdgcn_readlane(l * PER + at, __builtin_ctzll(holders));
            } else {
                if (LPT == 64 || !one_each(holders)) {
                    const uint32_t ml = lanes_max<LPT>(holds ? bl : 0u);
                    holds = holds && bl == ml;
                }
                // the lowest index as the largest of its complements
                e = ~lanes_max<LPT>(holds ? ~(l * PER + at) : 0u);
            }
#pragma unroll
            for (int k = 0; k < PER; ++k)
                key[k] = l * PER + k == e ? 0 : key[k];
            my_e = l == i ? e : my_e;
        }
        wave_lds_sync();
        // (top_k is at most the open experts, so every round found one)
        double w = l < p.top_k ? mine[min(my_e, uint32_t(p.experts - 1))] : 0.0;
        if (p.renormalize) {
            // summed in the order of choice
            double total = 0.0;
            for (int i = 0; i < p.top_k; ++i) total += lane_of(w, lane - l + i);
            w /= total;
        }
        wave_lds_sync();
        if (there && l < p.top_k) {
            const int64_t at = int64_t(t) * p.top_k + l;
            __hip_atomic_store(p.chosen + at, live ? int(my_e) : -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            p.weights[at] = live ? float(w * p.scale) : 0.f;
            if (p.segments) {
                if (live) atomicAdd(seg_counts + my_e, 1);
            } else if (one) {
                few[at] = live ? uint16_t(my_e) : kNoExpert;
            }
        }
    }
    if (p.segments) {
        __syncthreads();
        for (int e = tid; e < p.experts_up; e += kRouteThreads) p.counts[int64_t(blockIdx.x) * p.experts_up + e] = seg_counts[e];
        return;
    }
    const int n = p.tokens * p.top_k;
    if (one) {
        __syncthreads();
        order_few(p, few, n);
        return;
    }
    // the last workgroup orders the pairs
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (tid == 0) last = arrive(p.arrived, gridDim.x) ? 1 : 0;
    __syncthreads();
    if (!last) return;
    uint16_t* const choices = reinterpret_cast<uint16_t*>(route_lds);
#pragma unroll 4
    for (int i = tid; i < n; i += kRouteThreads)
        choices[i] = uint16_t(__hip_atomic_load(p.chosen + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
    __syncthreads();
    order_all(p, choices, n, reinterpret_cast<int*>(route_lds + kOneLaunch * 2));
}

// The pairs of the tokens of workgroup `seg` of the first launch to their places, behind those of the workgroups before it.
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(const RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t route_lds[];
    const int tid = threadIdx.x, seg = blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int* const base = reinterpret_cast<int*>(route_lds);
    int* const all = base + p.experts_up;
    int* const counts = all + p.experts_up;
    uint16_t* const choices = reinterpret_cast<uint16_t*>(counts + kRouteWaves * p.experts);
    for (int e = tid; e < 2 * p.experts_up; e += kRouteThreads) base[e] = 0;
    __syncthreads();
    // the workgroups' counts, four experts a thread and as many rows at once as there are threads for
    const int quads = p.experts_up / 4, at_once = kRouteThreads / quads;
    const int e0 = 4 * (tid % quads), row = tid / quads;
    if (row < at_once) {
        int4 a{0, 0, 0, 0}, b{0, 0, 0, 0};
#pragma unroll 8
        for (int k = row; k < p.segments; k += at_once) {
            const int4 v = *reinterpret_cast<const int4*>(p.counts + int64_t(k) * p.experts_up + e0);
            a = int4{a.x + v.x, a.y + v.y, a.z + v.z, a.w + v.w};
            if (k < seg) b = int4{b.x + v.x, b.y + v.y, b.z + v.z, b.w + v.w};
        }
        const int av[4] = {a.x, a.y, a.z, a.w}, bv[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            atomicAdd(all + e0 + i, av[i]);
            atomicAdd(base + e0 + i, bv[i]);
        }
    }
    __syncthreads();
    if (wave == 0) scan_experts(p, all, base, seg == 0 ? p.offsets : nullptr);
    const int64_t end = min(int64_t(seg + 1) * p.chunk, int64_t(p.tokens)) * p.top_k;
    for (int64_t begin = int64_t(seg) * p.chunk * p.top_k; begin < end; begin += kPiece) {
        const int n = static_cast<int>(min(end - begin, kPiece));
#pragma unroll 4
        for (int i = tid; i < n; i += kRouteThreads) choices[i] = uint16_t(p.chosen[begin + i]);
        int from, to;
        __syncthreads();
        count_piece(p, choices, n, counts, &from, &to);
        places_of_piece(p, counts, base);
        place_choices(p, choices, from, to, static_cast<int>(begin), counts + wave * p.experts);
        __syncthreads();
    }
}

__global__ void route_nothing_kernel(int32_t* offsets, int n) {
    const int i = blockIdx.x * kRouteThreads + threadIdx.x;
    if (i < n) offsets[i] = 0;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct RoutePlan {
    int lanes = 64;           // of a token
    int chunk = kRouteWaves;  // tokens of a workgroup
    int segments = 0;
    int64_t grid = 0;
    size_t ws_bytes = 0;
};

nmm_status plan_route(const nmm_moe_router& a, RoutePlan* q) {
    const int64_t lim = int64_t(1) << 26;
    if (a.tokens < 0 || a.tokens >= lim || a.experts < 1 || a.experts > kMaxRouted || a.top_k < 1 || a.top_k > 32 ||
        a.tokens * a.top_k >= lim)
        return NMM_ERR_SHAPE;
    if (a.groups < 1 || a.groups > 64 || a.experts % a.groups || a.top_groups < 1 || a.top_groups > a.groups ||
        a.top_k > a.experts / a.groups * a.top_groups)
        return NMM_ERR_SHAPE;
    *q = RoutePlan{};
    if (a.tokens * a.top_k > kOneLaunch) {
        // (60 experts, 512 tokens 10.3 us by 16 lanes and 9.1 by 64, 2048 10.9 and 11.1, 32767 22.3 and 33.0; 128 experts, 512 tokens 13.3
        // and 10.6, 8192 15.7 and 20.0.  More experts would be more than 8 of them a lane, more groups or choices more than its lanes.)
        if (a.tokens >= kSharedWaves && a.experts <= 128 && a.groups <= 16 && a.top_k <= 16) q->lanes = 16;
        const int64_t whole = kRouteWaves * (64 / q->lanes);
        q->chunk = static_cast<int>(cdiv(cdiv(a.tokens, max_segments(a.experts)), whole) * whole);
        q->segments = static_cast<int>(cdiv(a.tokens, q->chunk));
        q->ws_bytes = size_t(kTicketBytes) + size_t(q->segments) * (cdiv(a.experts, 4) * 4) * 4;
    } else if (a.tokens > kRouteWaves) {
        q->ws_bytes = size_t(kTicketBytes);
    }
    q->grid = cdiv(a.tokens, q->chunk);
    return NMM_OK;
}

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_moe_route_workspace_size(const nmm_moe_router* router) {
    RoutePlan q;
    return router && plan_route(*router, &q) == NMM_OK ? q.ws_bytes : 0;
}

nmm_status nmm_moe_route(const nmm_moe_router* router, void* workspace, size_t workspace_bytes, void* stream) {
    if (!router) return NMM_ERR_NULL;
    const nmm_moe_router& a = *router;
    if (a.logits_type != NMM_SRC_F32 && a.logits_type != NMM_SRC_BF16) return NMM_ERR_DTYPE;
    RoutePlan q;
    nmm_status st = plan_route(a, &q);
    if (st != NMM_OK) return st;
    if (a.ld_logits < a.experts || a.ld_logits >= (int64_t(1) << 31)) return NMM_ERR_SHAPE;
    if ((a.score != NMM_SCORE_SOFTMAX && a.score != NMM_SCORE_SIGMOID) || (a.group_top != 1 && a.group_top != 2) ||
        a.renormalize < 0 || a.renormalize > 1 || !std::isfinite(a.scale))
        return NMM_ERR_ARG;
    if (!a.offsets) return NMM_ERR_NULL;
    if (!aligned(a.offsets, 4)) return NMM_ERR_ALIGN;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const dim3 block(kRouteThreads);
    if (a.tokens == 0) {
        const int n = static_cast<int>(a.experts + 1);
        hipLaunchKernelGGL(route_nothing_kernel, dim3(cdiv(n, kRouteThreads)), block, 0, s, a.offsets, n);
        return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
    }
    if (!a.logits || !a.chosen || !a.weights || !a.pairs) return NMM_ERR_NULL;
    if (!aligned(a.logits, a.logits_type == NMM_SRC_F32 ? 4 : 2) || !aligned(a.bias, 4) || !aligned(a.chosen, 4) ||
        !aligned(a.weights, 4) || !aligned(a.pairs, 4))
        return NMM_ERR_ALIGN;
    st = validate_workspace(workspace, workspace_bytes, q.ws_bytes);
    if (st != NMM_OK) return st;
    RouteParams p{};
    p.logits = a.logits;
    p.ld = a.ld_logits;
    p.bias = a.bias;
    p.mask = a.mask;
    p.chosen = a.chosen;
    p.weights = a.weights;
    p.offsets = a.offsets;
    p.pairs = a.pairs;
    p.arrived = static_cast<unsigned*>(workspace);
    p.counts = q.segments ? reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + kTicketBytes) : nullptr;
    p.scale = double(a.scale);
    p.tokens = static_cast<int>(a.tokens);
    p.experts = static_cast<int>(a.experts);
    p.top_k = static_cast<int>(a.top_k);
    p.groups = static_cast<int>(a.groups);
    p.group_size = static_cast<int>(a.experts / a.groups);
    p.top_groups = static_cast<int>(a.top_groups);
    p.group_top = static_cast<int>(a.group_top);
    p.bf16 = a.logits_type == NMM_SRC_BF16;
    p.sigmoid = a.score == NMM_SCORE_SIGMOID;
    p.renormalize = a.renormalize;
    p.segments = q.segments;
    p.chunk = q.chunk;
    p.experts_up = static_cast<int>(cdiv(a.experts, 4) * 4);
    p.group_lanes = 1;
    while (p.group_lanes * 2 * p.groups <= q.lanes && p.group_lanes < 32) p.group_lanes *= 2;
    const int64_t bytes = p.bf16 ? 2 : 4;
    p.wide = a.experts % 4 == 0 && aligned(a.logits, 4 * bytes) && a.ld_logits % 4 == 0;
    const dim3 grid(static_cast<uint32_t>(q.grid));
    const size_t e4 = size_t(p.experts) * 4;
    size_t lds = size_t(kRouteWaves) * (64 / q.lanes) * p.experts * 8;
    lds = q.segments ? lds + p.experts_up * 4 : (q.grid > 1 ? std::max(lds, size_t(kOneLaunch) * 2 + e4 * (kRouteWaves + 2)) : lds);
    if (q.lanes == 16) {
        if (p.experts <= 64) hipLaunchKernelGGL((route_kernel<16, 4>), grid, block, lds, s, p);
        else hipLaunchKernelGGL((route_kernel<16, 8>), grid, block, lds, s, p);
    } else {
        if (p.experts <= 64) hipLaunchKernelGGL((route_kernel<64, 1>), grid, block, lds, s, p);
        else if (p.experts <= 128) hipLaunchKernelGGL((route_kernel<64, 2>), grid, block, lds, s, p);
        else if (p.experts <= 256) hipLaunchKernelGGL((route_kernel<64, 4>), grid, block, lds, s, p);
        else if (p.experts <= 512) hipLaunchKernelGGL((route_kernel<64, 8>), grid, block, lds, s, p);
        else hipLaunchKernelGGL((route_kernel<64, 16>), grid, block, lds, s, p);
    }
    if (q.segments)
        hipLaunchKernelGGL(route_place_kernel, grid, block,
                           size_t(p.experts_up) * 8 + e4 * kRouteWaves + size_t(kPiece) * 2, s, p);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
