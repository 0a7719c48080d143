// The chosen experts' products and their weighted sum: three launches.
//   up       h[s] = dt(act(x[t] Wg^T) * (x[t] Wu^T))       s: the pairs in the order by experts, t = pairs[s] / top_k
//   down     part[p] = h[s] W2^T, p = pairs[s]              fp32
//   combine  y[t] = dt(residual[t] + sum_i weights[t,i] part[t top_k + i])      in the order of i
// part is kept in 32 bits and added in order, so that results do not depend on which workgroup ends first (atomics would).  h is rounded
// to 16 bits, by choice: two words of them would keep its 32-bit value, at twice the bytes of h, LDS for it and reads of its fragments, and
// twice the matrix instructions, where wide tiles take as long to read fragments as to multiply them and 256 rows leave no LDS.  The
// rounding is half a step of each h, so y is off by at most about what its own rounding may be (bf16, no residual, 2.1e-3 to 2.4e-3 of y
// in the 2-norm against 1.6e-3 to 1.7e-3 with h in 32 bits; fp16 2.3e-4 to 3.0e-4 against 2.1e-4).
//
// What bounds it: the chosen experts' weights, each read once.  Hidden 7168, inner 2048: one token's 8 experts (705 MB) 119 us in the
// three launches, 64 tokens on 64 experts (5.6 GB) 915 to 960, 1024 tokens on the 16 of 64 experts that are here (1.4 GB, and 180 GFLOP)
// 382 to 399; of these up 67 to 69, 581 to 630, 226, down 45, 328 to 338, 132.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "moe_tiles.h"
#include "nmm_internal.h"
#include "nt_rows.h"
#include "nt_wide.h"

namespace nmm {
namespace {

using rows::RowsParams;
using ring::f32x4;

constexpr int64_t kLim = int64_t(1) << 31;
constexpr int kGridMost = 2048;            // workgroups: more items than that are taken in turns
constexpr int kCombineThreads = 256;
constexpr int64_t kCombineGridMost = int64_t(1) << 23;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t rup(int64_t a, int64_t b) { return cdiv(a, b) * b; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

struct CombineParams {
    const float* part;
    int64_t ld_part;
    const int32_t* chosen;
    const float* weights;
    const uint16_t* res;     // or NULL
    int64_t ldr;
    uint16_t* y;
    int64_t ldy;
    int tokens, top_k, first, local, N, col_blocks;
};

// Four columns of a token a thread; eight of its experts' sums are under way at a time.
template <int DT>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(const CombineParams p) {
    const int t = static_cast<int>(blockIdx.x / unsigned(p.col_blocks));
    const int n = (static_cast<int>(blockIdx.x % unsigned(p.col_blocks)) * kCombineThreads + int(threadIdx.x)) * 4;
    if (n >= p.N) return;
    f32x4 a{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < p.top_k; i0 += 8) {
        f32x4 s[8];
        float w[8];
        bool here[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t pair = int64_t(t) * p.top_k + min(i0 + j, p.top_k - 1);
            here[j] = i0 + j < p.top_k && uint32_t(p.chosen[pair] - p.first) < uint32_t(p.local);
            w[j] = p.weights[pair];
            // (the sums of a pair whose expert is elsewhere were not written)
            s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (here[j]) s[j] = *reinterpret_cast<const f32x4*>(p.part + pair * p.ld_part + n);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (here[j]) a += w[j] * s[j];
    }
    float v[4] = {a[0], a[1], a[2], a[3]};
    if (p.res) {
        const uint16_t* r = p.res + int64_t(t) * p.ldr + n;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) v[i] += rows::up16<DT>(r[i]);
    }
    rows::store4<DT>(p.y + int64_t(t) * p.ldy, n, p.N, v);
}

// A launch has fewer than 2^32 threads: of more tokens than that, as many as go in one after the other.  (A loop in the kernel
// instead took 1.3 us more for one token of 8 experts and 6 for 1024 tokens on 16 of 64.)
template <int DT>
void launch_combine(CombineParams c, hipStream_t s) {
    const int most = static_cast<int>(std::max<int64_t>(1, kCombineGridMost / c.col_blocks));
    for (int left = c.tokens; left > 0; left -= most) {
        c.tokens = std::min(left, most);
        hipLaunchKernelGGL((combine_kernel<DT>), dim3(static_cast<uint32_t>(c.tokens) * c.col_blocks), dim3(kCombineThreads), 0, s, c);
        const int64_t n = c.tokens, pairs = n * c.top_k;
        c.part = c.part ? c.part + pairs * c.ld_part : nullptr;
        c.chosen += pairs;
        c.weights += pairs;
        c.res = c.res ? c.res + n * c.ldr : nullptr;
        c.y += n * c.ldy;
    }
}

struct FfnPlan {
    int64_t pairs, ld_h, ld_part;
    size_t part_at, ws_bytes;
};

// Sizes that a call may have, and the workspace they need.
nmm_status plan_ffn(const nmm_moe_ffn& a, FfnPlan* q) {
    if (a.tokens < 0 || a.top_k < 1 || a.top_k > 32 || a.experts < 1 || a.experts > rows::kMaxExperts) return NMM_ERR_SHAPE;
    if (a.tokens >= (int64_t(1) << 26) || a.tokens * a.top_k >= (int64_t(1) << 26)) return NMM_ERR_SHAPE;
    if (a.first < 0 || a.local < 0 || a.first > a.experts || a.local > a.experts - a.first) return NMM_ERR_SHAPE;
    if (a.hidden < 1 || a.inner < 1 || a.hidden >= kLim / 4 || a.inner >= kLim / 4) return NMM_ERR_SHAPE;
    q->pairs = a.tokens * a.top_k;
    q->ld_h = rup(a.inner, 64);
    q->ld_part = rup(a.hidden, 4);
    if (a.local == 0) {
        q->part_at = q->ws_bytes = 0;
        return NMM_OK;
    }
    q->part_at = size_t(kTicketBytes) + size_t(rup(q->pairs * q->ld_h * 2, 256));
    q->ws_bytes = q->pairs ? q->part_at + size_t(q->pairs) * q->ld_part * 4 : 0;
    return NMM_OK;
}

// Workgroups of a launch whose tiles have `rows` rows of x: a cut tile per expert that has pairs, and whole ones.
uint32_t grid_of(const RowsParams& p, int64_t pairs, int64_t rows) {
    const int64_t tiles = std::min<int64_t>(p.local, pairs) + pairs / rows;
    return static_cast<uint32_t>(std::min<int64_t>(cdiv(p.n_blocks, 8) * 8 * tiles, kGridMost));
}

// 32 rows of the weight and two waves a workgroup, of which three share a CU up to 8 rows of x (45 to 49 KB of LDS) and two at 16 (57 KB): the
// eight experts of one token, W2 44.9 us (52.2 with four waves, whose workgroups have a CU each).  Up to 8 rows of x and a K of eight groups
// for each of four waves W1 goes by 16 rows, a gate's 8 and the 8 that it multiplies: 67.4 us of one token (73.0 in 32s), 41 of four experts of 4096 x 4096 (58); at 16 rows of x 439 and 432.
template <int DT, int MODE, int XR>
void launch_few(RowsParams p, int64_t pairs, hipStream_t s) {
    if constexpr (MODE == rows::kUp && XR <= 2) {
        if (p.K >= 4 * 8 * kMfmaNtGroup) {
            p.n_blocks = static_cast<int>(cdiv(p.N, 8));
            hipLaunchKernelGGL((rows::rows_kernel<DT, MODE, XR, 1, 4>), dim3(grid_of(p, pairs, 4 * XR)), dim3(256), 0, s, p);
            return;
        }
    }
    p.n_blocks = static_cast<int>(cdiv(p.N, MODE == rows::kUp ? 16 : 32));
    hipLaunchKernelGGL((rows::rows_kernel<DT, MODE, XR, 2, 2>), dim3(grid_of(p, pairs, 4 * XR)), dim3(128), 0, s, p);
}

template <int DT, int MODE, int BM>
void launch_wide(RowsParams p, int64_t pairs, hipStream_t s) {
    constexpr int BN = 128;
    p.n_blocks = static_cast<int>(cdiv(p.N, MODE == rows::kUp ? BN / 2 : BN));
    hipLaunchKernelGGL((rows::wide_kernel<DT, MODE, BM, BN, 3>), dim3(grid_of(p, pairs, BM)), dim3(rows::kWideThreads), 0, s, p);
}

template <int DT, int MODE>
void launch_rows(const RowsParams& p, int tile_rows, int64_t pairs, hipStream_t s) {
    switch (tile_rows) {
        case 4: return launch_few<DT, MODE, 1>(p, pairs, s);
        case 8: return launch_few<DT, MODE, 2>(p, pairs, s);
        case 16: return launch_few<DT, MODE, 4>(p, pairs, s);
        case 64: return launch_wide<DT, MODE, 64>(p, pairs, s);
        case 128: return launch_wide<DT, MODE, 128>(p, pairs, s);
        default: return launch_wide<DT, MODE, 256>(p, pairs, s);
    }
}

template <int DT>
void launch(const RowsParams& up, const RowsParams& down, const CombineParams& c, const nmm_moe_ffn& a, int64_t pairs,
            hipStream_t s) {
    if (a.local > 0) {
        // (the first product's rows are addressed from x on, which is below 2^31 bytes)
        launch_rows<DT, rows::kUp>(up, rows::tile_rows_of(up.K, up.N, a.tokens, pairs, a.experts, a.local), pairs, s);
        launch_rows<DT, rows::kDown>(
            down, rows::tile_rows_in_reach(down.K, down.N, a.tokens, pairs, a.experts, a.local, down.ldx), pairs, s);
    }
    launch_combine<DT>(c, s);
}

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_moe_experts_workspace_size(const nmm_moe_ffn* ffn) {
    FfnPlan q;
    return ffn && plan_ffn(*ffn, &q) == NMM_OK ? q.ws_bytes : 0;
}

nmm_status nmm_moe_experts(const nmm_moe_ffn* ffn, void* workspace, size_t workspace_bytes, void* stream) {
    if (!ffn) return NMM_ERR_NULL;
    const nmm_moe_ffn& a = *ffn;
    if (a.dt != NMM_F16 && a.dt != NMM_BF16) return NMM_ERR_DTYPE;
    if (a.act < NMM_ACT_NONE || a.act > NMM_ACT_GELU_TANH) return NMM_ERR_ARG;
    FfnPlan q;
    nmm_status st = plan_ffn(a, &q);
    if (st != NMM_OK) return st;
    if (a.tokens == 0) return NMM_OK;
    if (!a.x || !a.chosen || !a.weights || !a.offsets || !a.pairs || !a.y) return NMM_ERR_NULL;
    if (a.ldx < a.hidden || a.ldx >= kLim || a.ldy < a.hidden || a.ldy >= kLim) return NMM_ERR_SHAPE;
    if (a.residual && (a.ldr < a.hidden || a.ldr >= kLim)) return NMM_ERR_SHAPE;
    if (!aligned(a.x, 16) || a.ldx % 8 || !aligned(a.y, 2) || !aligned(a.residual, 2) || !aligned(a.chosen, 4) ||
        !aligned(a.weights, 4) || !aligned(a.offsets, 4) || !aligned(a.pairs, 4))
        return NMM_ERR_ALIGN;
    // buffer offsets are 32-bit: x, and one expert's matrices
    const int64_t h8 = rup(a.hidden, 8), i8 = rup(a.inner, 8);
    if (((a.tokens - 1) * a.ldx + h8) * 2 >= kLim) return NMM_ERR_SHAPE;
    int64_t extent1 = 0, extent2 = 0;
    if (a.local > 0) {
        if (!a.W1 || !a.W2) return NMM_ERR_NULL;
        if (a.ldw1 < a.hidden || a.ldw1 >= kLim || a.ldw2 < a.inner || a.ldw2 >= kLim) return NMM_ERR_SHAPE;
        extent1 = (2 * a.inner - 1) * a.ldw1 + h8;
        extent2 = (a.hidden - 1) * a.ldw2 + i8;
        if (extent1 * 2 >= kLim || extent2 * 2 >= kLim) return NMM_ERR_SHAPE;
        const int64_t far = int64_t(1) << 50;
        if (a.local > 1 && (a.stride1 < (2 * a.inner - 1) * a.ldw1 + a.hidden || a.stride2 < (a.hidden - 1) * a.ldw2 + a.inner ||
                            a.stride1 >= far || a.stride2 >= far))
            return NMM_ERR_SHAPE;
        if (!aligned(a.W1, 16) || !aligned(a.W2, 16) || a.ldw1 % 8 || a.ldw2 % 8 || (a.local > 1 && (a.stride1 % 8 || a.stride2 % 8)))
            return NMM_ERR_ALIGN;
    }
    const bool in_place = a.residual && a.residual == a.y && a.ldr == a.ldy;
    if ((!in_place && rows_overlap(a.residual, 2 * a.ldr, 2 * a.hidden, a.y, 2 * a.ldy, 2 * a.hidden, a.tokens)) ||
        rows_overlap(a.x, 2 * a.ldx, 2 * a.hidden, a.y, 2 * a.ldy, 2 * a.hidden, a.tokens))
        return NMM_ERR_ARG;
    CombineParams c{};
    c.col_blocks = static_cast<int>(cdiv(a.hidden, 4 * kCombineThreads));
    st = validate_workspace(workspace, workspace_bytes, q.ws_bytes);
    if (st != NMM_OK) return st;
    RowsParams up{}, down{};
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    up.local = down.local = static_cast<int>(a.local);
    up.top_k = down.top_k = static_cast<int>(a.top_k);
    up.M = down.M = static_cast<int>(q.pairs);
    up.offsets = down.offsets = a.offsets + a.first;
    up.pairs = down.pairs = a.pairs;
    up.act = a.act;
    up.ks = down.ks = 1;
    up.rot = rows::rotation(a.ldw1);
    down.rot = rows::rotation(a.ldw2);
    if (a.local > 0) {
        uint16_t* const h = reinterpret_cast<uint16_t*>(ws + kTicketBytes);
        float* const part = reinterpret_cast<float*>(ws + q.part_at);
        up.x = static_cast<const uint16_t*>(a.x);
        up.ldx = a.ldx;
        up.x_extent = static_cast<uint32_t>(((a.tokens - 1) * a.ldx + h8) * 2);
        up.w = static_cast<const uint8_t*>(a.W1);
        up.w_stride = a.local > 1 ? a.stride1 * 2 : 0;
        up.row_bytes = static_cast<uint32_t>(a.ldw1 * 2);
        up.w_extent = static_cast<uint32_t>(extent1 * 2);
        up.K = static_cast<int>(a.hidden);
        up.N = static_cast<int>(a.inner);
        up.y = h;
        up.ldy = q.ld_h;
        down.x = h;
        down.ldx = q.ld_h;
        down.w = static_cast<const uint8_t*>(a.W2);
        down.w_stride = a.local > 1 ? a.stride2 * 2 : 0;
        down.row_bytes = static_cast<uint32_t>(a.ldw2 * 2);
        down.w_extent = static_cast<uint32_t>(extent2 * 2);
        down.K = static_cast<int>(a.inner);
        down.N = static_cast<int>(a.hidden);
        down.yf = part;
        down.ldyf = q.ld_part;
        c.part = part;
        c.ld_part = q.ld_part;
    }
    c.chosen = a.chosen;
    c.weights = a.weights;
    c.res = static_cast<const uint16_t*>(a.residual);
    c.ldr = a.ldr;
    c.y = static_cast<uint16_t*>(a.y);
    c.ldy = a.ldy;
    c.tokens = static_cast<int>(a.tokens);
    c.top_k = static_cast<int>(a.top_k);
    c.first = static_cast<int>(a.first);
    c.local = static_cast<int>(a.local);
    c.N = static_cast<int>(a.hidden);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.dt == NMM_BF16) launch<NMM_BF16>(up, down, c, a, q.pairs, s);
    else launch<NMM_F16>(up, down, c, a, q.pairs, s);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
