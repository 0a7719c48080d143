// Routing to experts: scores, the choice of each token, and the (token, expert) pairs in the order of the experts.
//
// A wave takes a token, lane l the experts l PER .. l PER + PER - 1, all in fp64: which expert comes before which may not
// depend on how a score was rounded.  Choosing is top_k rounds of a wave maximum; the first lane that holds it has the
// lowest index, and what has been chosen or lies in a closed group becomes NaN, which a maximum passes over.
//
// The pairs are sorted by counting: a wave walks its stretch of pairs, 64 at a time, and learns from one ballot per bit of the
// expert's number which lanes hold the same one, so that a pair's place is its expert's next place plus its rank among them.
// Up to kOneLaunch pairs the last workgroup to finish its tokens does it (handoff.h), more take two launches over segments.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "handoff.h"
#include "nmm_internal.h"
#include "wave64.h"

namespace nmm {
namespace {

constexpr int kRouteThreads = 256, kRouteWaves = kRouteThreads / 64;
constexpr int64_t kOneLaunch = 8192;
constexpr int kMaxSegments = 64;
constexpr int kRouteGridMost = 65536;
constexpr int kMaxRouted = 1024;      // experts

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
    int32_t* counts;          // [segments][experts], more than kOneLaunch pairs
    double scale;
    int tokens, experts, top_k;
    int groups, group_size, top_groups, group_top;
    int bf16, sigmoid, renormalize;
    int segments;             // 0: the pairs are ordered in the first launch
    int segment;              // pairs of one
};

__device__ __forceinline__ double readlane64(double x, int lane) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(u)), lane), hi = __builtin_amdgcn_readlane(int(uint32_t(u >> 32)), lane);
    return __longlong_as_double((uint64_t(hi) << 32) | lo);
}

// LDS of a wave written by some of its lanes and read by others.
__device__ __forceinline__ void wave_lds_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ int load_choice(const RouteParams& p, int64_t pair) {
    return __hip_atomic_load(p.chosen + pair, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Counts of the experts in pairs begin .. end of this wave.
__device__ __forceinline__ void count_pairs(const RouteParams& p, int64_t begin, int64_t end, int* counts) {
    for (int64_t i = begin + (threadIdx.x & 63); i < end; i += 64) {
        const int e = load_choice(p, i);
        if (e >= 0) atomicAdd(counts + e, 1);
    }
}

// Pairs begin .. end of this wave to their places; next[e]: the next place of expert e.
__device__ __forceinline__ void place_pairs(const RouteParams& p, int64_t begin, int64_t end, int* next) {
    const int lane = threadIdx.x & 63;
    const int bits = 32 - __builtin_clz(p.experts);
    for (int64_t i0 = begin; i0 < end; i0 += 64) {
        const int64_t i = i0 + lane;
        const int e = i < end ? load_choice(p, i) : -1;
        uint64_t same = __builtin_amdgcn_ballot_w64(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t ones = __builtin_amdgcn_ballot_w64((e >> b) & 1);
            same &= (e >> b) & 1 ? ones : ~ones;
        }
        if (e >= 0) {
            const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
            const int at = next[e];
            p.pairs[at + rank] = static_cast<int32_t>(i);
            wave_lds_sync();
            if (rank == 0) next[e] = at + __builtin_popcountll(same);
        }
        wave_lds_sync();
    }
}

// counts[w][e] of the four waves become their next places, given `before` pairs of expert e ahead of them (segments) and
// `all` of it in total: an exclusive sum over the experts.  By the first wave.  Where `offsets` is given, it is written.
template <class Before, class All>
__device__ __forceinline__ void places_of(const RouteParams& p, int* counts, Before before, All all, int32_t* offsets) {
    const int lane = threadIdx.x & 63;
    int carry = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const int e = e0 + lane;
        const int mine = e < p.experts ? all(e) : 0;
        int c = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(c, d);
            if (lane >= d) c += o;
        }
        if (e < p.experts) {
            const int start = carry + c - mine;
            if (offsets) offsets[e] = start;
            int at = start + before(e);
#pragma unroll
            for (int w = 0; w < kRouteWaves; ++w) {
                const int n = counts[w * p.experts + e];
                counts[w * p.experts + e] = at;
                at += n;
            }
        }
        carry += __shfl(c, 63);
    }
    if (offsets && lane == 0) offsets[p.experts] = carry;
}

// Pairs begin .. end, the waves a stretch of whole 64s each.
__device__ __forceinline__ void stretch_of(int64_t begin, int64_t end, int wave, int64_t* from, int64_t* to) {
    const int64_t each = ((end - begin + 64 * kRouteWaves - 1) / (64 * kRouteWaves)) * 64;
    *from = begin + wave * each < end ? begin + wave * each : end;
    *to = *from + each < end ? *from + each : end;
}

template <int PER>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(const RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t route_lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const double nan = __longlong_as_double(0x7FF8000000000000ll);
    double* const group_c = reinterpret_cast<double*>(route_lds) + wave * p.experts;
    for (int t = static_cast<int>(blockIdx.x) * kRouteWaves + wave; t < p.tokens; t += static_cast<int>(gridDim.x) * kRouteWaves) {
        const int64_t out = int64_t(t) * p.top_k;
        if (p.mask && p.mask[t] == 0) {
            if (lane < p.top_k) {
                __hip_atomic_store(p.chosen + out + lane, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                p.weights[out + lane] = 0.f;
            }
            continue;
        }
        double s[PER], c[PER];
        const int64_t row = int64_t(t) * p.ld;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane * PER + i;
            s[i] = nan;
            if (e < p.experts)
                s[i] = p.bf16 ? double(__uint_as_float(uint32_t(static_cast<const uint16_t*>(p.logits)[row + e]) << 16))
                              : double(static_cast<const float*>(p.logits)[row + e]);
        }
        if (p.sigmoid) {
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] = 1.0 / (1.0 + exp(-s[i]));
        } else {
            double top = s[0], sum = 0.0;
#pragma unroll
            for (int i = 1; i < PER; ++i) top = __builtin_fmax(top, s[i]);
            top = max64(top);
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                s[i] = exp(s[i] - top);
                if (lane * PER + i < p.experts) sum += s[i];
            }
            sum = sum64(sum);
#pragma unroll
            for (int i = 0; i < PER; ++i) s[i] /= sum;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane * PER + i;
            c[i] = nan;
            if (e < p.experts) {
                c[i] = p.bias ? s[i] + double(p.bias[e]) : s[i];
                if (c[i] != c[i]) c[i] = -INFINITY;
            }
        }
        if (p.groups > 1) {
            // lane g takes group g's best one or two, then its rank among the groups
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (lane * PER + i < p.experts) group_c[lane * PER + i] = c[i];
            wave_lds_sync();
            double best = -INFINITY, second = -INFINITY;
            if (lane < p.groups)
                for (int i = 0; i < p.group_size; ++i) {
                    const double v = group_c[lane * p.group_size + i];
                    second = v > best ? best : (v > second ? v : second);
                    best = v > best ? v : best;
                }
            wave_lds_sync();
            double total = p.group_top == 2 && p.group_size > 1 ? best + second : best;
            if (total != total) total = -INFINITY;
            int ahead = 0;
            for (int o = 0; o < p.groups; ++o) {
                const double v = readlane64(total, o);
                ahead += v > total || (v == total && o < lane) ? 1 : 0;
            }
            const uint64_t open = __builtin_amdgcn_ballot_w64(lane < p.groups && ahead < p.top_groups);
            int grp = lane * PER / p.group_size, left = (grp + 1) * p.group_size - lane * PER;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (left == 0) {
                    ++grp;
                    left = p.group_size;
                }
                if (grp < 64 && !((open >> grp) & 1)) c[i] = nan;
                --left;
            }
        }
        int my_e = 0;
        double my_s = 0.0, total = 0.0;
        for (int i = 0; i < p.top_k; ++i) {
            double top = c[0];
#pragma unroll
            for (int k = 1; k < PER; ++k) top = __builtin_fmax(top, c[k]);
            top = max64(top);
            int at = PER;
            double sv = 0.0;
#pragma unroll
            for (int k = PER - 1; k >= 0; --k)
                if (c[k] == top) {
                    at = k;
                    sv = s[k];
                }
            const uint64_t holders = __builtin_amdgcn_ballot_w64(at < PER);
            const int first = __builtin_ctzll(holders);       // (top_k is at most the open experts, so there is one)
            const int e = __builtin_amdgcn_readlane(lane * PER + at, first);
            const double v = readlane64(sv, first);
            total += v;
            if (lane == first) {
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (k == at) c[k] = nan;
            }
            if (lane == i) {
                my_e = e;
                my_s = v;
            }
        }
        if (lane < p.top_k) {
            __hip_atomic_store(p.chosen + out + lane, my_e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            p.weights[out + lane] = float((p.renormalize ? my_s / total : my_s) * p.scale);
        }
    }
    if (p.segments) return;
    // the last workgroup orders the pairs
    __shared__ int last;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (gridDim.x > 1) {
        if (tid == 0) last = arrive(p.arrived, gridDim.x) ? 1 : 0;
        __syncthreads();
        if (!last) return;
    }
    int* const counts = reinterpret_cast<int*>(route_lds);
    for (int i = tid; i < kRouteWaves * p.experts; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    int64_t from, to;
    stretch_of(0, int64_t(p.tokens) * p.top_k, wave, &from, &to);
    count_pairs(p, from, to, counts + wave * p.experts);
    __syncthreads();
    if (wave == 0)
        places_of(p, counts, [](int) { return 0; },
                  [&](int e) {
                      int n = 0;
#pragma unroll
                      for (int w = 0; w < kRouteWaves; ++w) n += counts[w * p.experts + e];
                      return n;
                  },
                  p.offsets);
    __syncthreads();
    place_pairs(p, from, to, counts + wave * p.experts);
}

// Counts of a segment of pairs.
__global__ __launch_bounds__(kRouteThreads) void route_count_kernel(const RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t route_lds[];
    int* const counts = reinterpret_cast<int*>(route_lds);
    const int tid = threadIdx.x;
    for (int i = tid; i < p.experts; i += kRouteThreads) counts[i] = 0;
    __syncthreads();
    const int64_t n = int64_t(p.tokens) * p.top_k, begin = int64_t(blockIdx.x) * p.segment;
    const int64_t end = begin + p.segment < n ? begin + p.segment : n;
    int64_t from, to;
    stretch_of(begin, end, tid >> 6, &from, &to);
    count_pairs(p, from, to, counts);
    __syncthreads();
    for (int i = tid; i < p.experts; i += kRouteThreads) p.counts[int64_t(blockIdx.x) * p.experts + i] = counts[i];
}

// A segment's pairs to their places, behind those of the segments before it.
__global__ __launch_bounds__(kRouteThreads) void route_place_kernel(const RouteParams p) {
    extern __shared__ __attribute__((aligned(16))) uint8_t route_lds[];
    int* const counts = reinterpret_cast<int*>(route_lds);
    int* const before = counts + kRouteWaves * p.experts;
    int* const all = before + p.experts;
    const int tid = threadIdx.x, wave = tid >> 6, seg = blockIdx.x;
    for (int i = tid; i < kRouteWaves * p.experts; i += kRouteThreads) counts[i] = 0;
    for (int e = tid; e < p.experts; e += kRouteThreads) {
        int b = 0, a = 0;
#pragma unroll 8
        for (int k = 0; k < p.segments; ++k) {
            const int v = p.counts[int64_t(k) * p.experts + e];
            a += v;
            b += k < seg ? v : 0;
        }
        before[e] = b;
        all[e] = a;
    }
    __syncthreads();
    const int64_t n = int64_t(p.tokens) * p.top_k, begin = int64_t(seg) * p.segment;
    const int64_t end = begin + p.segment < n ? begin + p.segment : n;
    int64_t from, to;
    stretch_of(begin, end, wave, &from, &to);
    count_pairs(p, from, to, counts + wave * p.experts);
    __syncthreads();
    if (wave == 0)
        places_of(p, counts, [&](int e) { return before[e]; }, [&](int e) { return all[e]; }, seg == 0 ? p.offsets : nullptr);
    __syncthreads();
    place_pairs(p, from, to, counts + wave * p.experts);
}

__global__ void route_nothing_kernel(int32_t* offsets, int n) {
    const int i = blockIdx.x * kRouteThreads + threadIdx.x;
    if (i < n) offsets[i] = 0;
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct RoutePlan {
    int segments = 0, segment = 0;
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
    const int64_t n = a.tokens * a.top_k;
    *q = RoutePlan{};
    if (n > kOneLaunch) {
        q->segment = static_cast<int>(std::max<int64_t>(1024, cdiv(cdiv(n, kMaxSegments), 64 * kRouteWaves) * 64 * kRouteWaves));
        q->segments = static_cast<int>(cdiv(n, q->segment));
        q->ws_bytes = size_t(kTicketBytes) + size_t(q->segments) * a.experts * 4;
    } else if (a.tokens > kRouteWaves) {
        q->ws_bytes = size_t(kTicketBytes);
    }
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
    p.segment = q.segment;
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(cdiv(a.tokens, kRouteWaves), kRouteGridMost)));
    const size_t lds = size_t(kRouteWaves) * p.experts * (p.groups > 1 ? 8 : 4);
    if (p.experts <= 64) hipLaunchKernelGGL((route_kernel<1>), grid, block, lds, s, p);
    else if (p.experts <= 128) hipLaunchKernelGGL((route_kernel<2>), grid, block, lds, s, p);
    else if (p.experts <= 256) hipLaunchKernelGGL((route_kernel<4>), grid, block, lds, s, p);
    else if (p.experts <= 512) hipLaunchKernelGGL((route_kernel<8>), grid, block, lds, s, p);
    else hipLaunchKernelGGL((route_kernel<16>), grid, block, lds, s, p);
    if (q.segments) {
        hipLaunchKernelGGL(route_count_kernel, dim3(q.segments), block, size_t(p.experts) * 4, s, p);
        hipLaunchKernelGGL(route_place_kernel, dim3(q.segments), block, size_t(p.experts) * 4 * (kRouteWaves + 2), s, p);
    }
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
