// The product with [N, K] weights and a feed-forward layer's epilogue (bias, activation, gate, residual) in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nmm_internal.h"
#include "nt_rows.h"
#include "nt_wide.h"

namespace nmm {
namespace {

using rows::RowsParams;

constexpr int64_t kLim = int64_t(1) << 31;
constexpr int kGridMost = 2048;            // workgroups: more items than that are taken in turns

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <int DT, int XR, int NT>
void launch_rows(RowsParams p, hipStream_t s) {
    constexpr int NW = 4, D = NT == 1 && XR < 4 ? 3 : 2;
    p.n_blocks = static_cast<int>(cdiv(p.N, p.gated ? 16 : 16 * NT));
    const int64_t items = cdiv(p.n_blocks, 8) * 8 * cdiv(p.M, 4 * XR);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(items, kGridMost))), block(64 * NW);
    hipLaunchKernelGGL((rows::rows_kernel<DT, rows::kDense, XR, NT, NW, D>), grid, block, 0, s, p);
}

template <int DT, int XR>
void launch_nt(const RowsParams& p, hipStream_t s) {
    if (p.gated || XR >= 4) launch_rows<DT, XR, 2>(p, s);
    else launch_rows<DT, XR, 1>(p, s);
}

template <int DT, int BM, int BN, int S>
void launch_wide(RowsParams p, hipStream_t s) {
    p.n_blocks = static_cast<int>(cdiv(p.N, p.gated ? BN / 2 : BN));
    const int64_t items = cdiv(p.n_blocks, 8) * 8 * cdiv(p.M, BM);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(items, kGridMost))), block(rows::kWideThreads);
    hipLaunchKernelGGL((rows::wide_kernel<DT, rows::kDense, BM, BN, S>), grid, block, 0, s, p);
}

template <int DT>
void launch(const RowsParams& p, hipStream_t s) {
    if (p.M <= 4) launch_nt<DT, 1>(p, s);
    else if (p.M <= 8) launch_nt<DT, 2>(p, s);
    else if (p.M <= 16) launch_nt<DT, 4>(p, s);
    else if (p.M <= 32) launch_nt<DT, 8>(p, s);
    else launch_wide<DT, 64, 64, 4>(p, s);
}

}  // namespace

bool rows_overlap(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb, int64_t n) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    if (!a || !b || n <= 0 || wa <= 0 || wb <= 0) return false;
    if (pa + uintptr_t((n - 1) * lda + wa) <= pb || pb + uintptr_t((n - 1) * ldb + wb) <= pa) return false;
    if (lda != ldb || n == 1) return true;
    const uintptr_t d = (pb >= pa ? pb - pa : uintptr_t(lda) - (pa - pb) % uintptr_t(lda)) % uintptr_t(lda);
    return d < uintptr_t(wa) || d + uintptr_t(wb) > uintptr_t(lda);
}

}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_gemv_nt_act_workspace_size(const nmm_nt_act*) { return 0; }

nmm_status nmm_gemv_nt_act(const nmm_nt_act* product, void*, size_t, void* stream) {
    if (!product) return NMM_ERR_NULL;
    const nmm_nt_act& a = *product;
    if (a.dt != NMM_F16 && a.dt != NMM_BF16) return NMM_ERR_DTYPE;
    if (a.M < 0 || a.K < 0 || a.N < 0 || a.M >= kLim || a.K >= kLim || a.N >= kLim) return NMM_ERR_SHAPE;
    if (a.act < NMM_ACT_NONE || a.act > NMM_ACT_GELU_TANH || a.gated < 0 || a.gated > 1) return NMM_ERR_ARG;
    if (a.M == 0 || a.N == 0) return NMM_OK;
    if (!a.y && !a.y_f32) return NMM_ERR_NULL;
    if (a.y && (a.ldy < a.N || a.ldy >= kLim)) return NMM_ERR_SHAPE;
    if (a.y_f32 && (a.ldyf < a.N || a.ldyf >= kLim)) return NMM_ERR_SHAPE;
    if (a.residual && (a.ldr < a.N || a.ldr >= kLim)) return NMM_ERR_SHAPE;
    if (!aligned(a.y, 2) || !aligned(a.y_f32, 4) || !aligned(a.bias, 2) || !aligned(a.residual, 2)) return NMM_ERR_ALIGN;
    const int64_t n_rows = a.gated ? 2 * a.N : a.N, k8 = cdiv(a.K, 8) * 8;
    if (n_rows >= kLim / 2) return NMM_ERR_SHAPE;
    if (a.K > 0) {
        if (!a.x || !a.Wt) return NMM_ERR_NULL;
        if (a.ldx < a.K || a.ldx >= kLim || a.ldwt < a.K || a.ldwt >= kLim) return NMM_ERR_SHAPE;
        if (!aligned(a.x, 16) || !aligned(a.Wt, 16) || a.ldx % 8 || a.ldwt % 8) return NMM_ERR_ALIGN;
        // buffer offsets are 32-bit: the weight, and the rows of x in a block
        if (((n_rows - 1) * a.ldwt + k8) * 2 >= kLim) return NMM_ERR_SHAPE;
        if (((std::min<int64_t>(a.M, 128) - 1) * a.ldx + k8) * 2 >= kLim) return NMM_ERR_SHAPE;
    }
    const bool in_place = a.residual && a.residual == a.y && a.ldr == a.ldy;
    if (!in_place && rows_overlap(a.residual, 2 * a.ldr, 2 * a.N, a.y, 2 * a.ldy, 2 * a.N, a.M)) return NMM_ERR_ARG;
    if (a.K > 0 && (rows_overlap(a.x, 2 * a.ldx, 2 * a.K, a.y, 2 * a.ldy, 2 * a.N, a.M) ||
                    rows_overlap(a.x, 2 * a.ldx, 2 * a.K, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M)))
        return NMM_ERR_ARG;
    if (rows_overlap(a.residual, 2 * a.ldr, 2 * a.N, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M) ||
        rows_overlap(a.y, 2 * a.ldy, 2 * a.N, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M))
        return NMM_ERR_ARG;
    RowsParams p{};
    p.x = static_cast<const uint16_t*>(a.x);
    if (a.K > 0) {             // (0: extents of nothing)
        p.ldx = a.ldx;
        p.w = static_cast<const uint8_t*>(a.Wt);
        p.row_bytes = static_cast<uint32_t>(a.ldwt * 2);
        p.w_extent = static_cast<uint32_t>(((n_rows - 1) * a.ldwt + k8) * 2);
    }
    p.K = static_cast<int>(a.K);
    p.N = static_cast<int>(a.N);
    p.M = static_cast<int>(a.M);
    p.gated = a.gated;
    p.act = a.act;
    p.bias = static_cast<const uint16_t*>(a.bias);
    p.res = static_cast<const uint16_t*>(a.residual);
    p.ldr = a.ldr;
    p.y = static_cast<uint16_t*>(a.y);
    p.ldy = a.ldy;
    p.yf = a.y_f32;
    p.ldyf = a.ldyf;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.dt == NMM_BF16) launch<NMM_BF16>(p, s);
    else launch<NMM_F16>(p, s);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
